// Products of 8-bit rows with 8-bit weights: the projections around the attention in a sampler.
//     y[m, n] = s[m] ws[n] sum_k q[m, k] w[n, k] + bias[n]
// q (M, K) with a scale for each row (token), w (N, K) with a scale for each row (output channel), both K-major; the sum is
// exact (32-bit integers), the rest is fp32 and rounded once to the output's type.
//
// Many rows: tcgen05.mma kind::i8 (32-bit integer accumulators in tensor memory) on pairs of CTAs, 256 rows x BN channels a
// tile.  An MMA of a pair reads half of the weights' tile from each CTA's shared memory: tiles of 128 x 256 on single CTAs would
// load 24 and read 12 KB where these load 16 and read 8, more than the 128 bytes a cycle that shared memory has at the rate of
// the tensor cores.  Warp 0 loads by TMA, warp 1 of the pair's first CTA issues the MMAs, warps 4 to 11 scale and store one
// accumulator while the other one fills; a pair walks over its tiles, and the ring of loads runs on through them.
//
// Up to 256 rows the weights' bytes are what a product costs.  There the weights can be the tensor cores' operand with 128 rows and stream past the
// tokens, the CTAs of a cluster sharing k; that is done where it is faster than tiles of 256 rows (14336 x 4096 weights: up to 57 tokens, 4096 x
// 14336: always; the rule and its times stand at linear() in row_ops_api.cu).  Up to 2 rows (single tokens) dp4a on operands that go from global memory
// straight to registers keeps pace with HBM: nothing is set up, and nothing waits.  (mma.sync, which emulates 8-bit products on this
// GPU at some 150 multiply-adds a cycle and SM, took 20 us for one token and 14336 x 4096 weights.)
//
// Measured on B200: 16384 x 3456 x 1152, bf16 out, 52 us in bursts and 61 at the power cap (2.1 Pop/s), 16384 x 4608 x 9216 421 (3.3 Pop/s, bursts), output
// alone (K = 128) at the rate of a fill; one token against 14336 x 4096 11.6 us (5 TB/s), 28672 x 4096 20.3 (5.8), 16 tokens 13.9; 64
// and 256 tokens, in tiles of 256 rows on 112 SMs, 17.5 and 18.
#pragma once
#include <cuda.h>
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
    int ksplit;                // some rows: CTAs of a cluster, which share k
    int tiles_m, tiles_n;      // many rows
    int tma_cols;              // columns of y that bulk stores may reach into: they write 16 bytes at a time, behind the end of a row too
    int* status;               // device status word; non-zero makes the kernel a no-op
};

template <typename T> __device__ __forceinline__ T linear_round(float v);
template <> __device__ __forceinline__ float linear_round<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 linear_round<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// ------------------------------------------------------------------------------------------------ few rows
constexpr int LIN_FEW_THREADS = 128, LIN_FEW_LOADS = 8;   // 16-byte loads of weights that a lane has in flight

// 16 bytes of a row of k, zeros behind its end (the memory behind it is not read).  (No loads by the read-only path in these kernels: they are
// set up while the kernel in front of them may still write what they read.)
__device__ __forceinline__ uint4 linear_load16(const int8_t* row, int k, int K, bool stream) {
    uint4 v = make_uint4(0, 0, 0, 0);
    if (k + 16 <= K) {
        if (stream) asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(row + k));
        else v = *reinterpret_cast<const uint4*>(row + k);
    } else if (k < K) {
        uint32_t b[4] = {0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < 16; ++j)
            if (k + j < K) b[j / 4] |= (uint32_t)(uint8_t)row[k + j] << (8 * (j & 3));
        v = make_uint4(b[0], b[1], b[2], b[3]);
    }
    return v;
}

// Up to MT tokens, R channels a warp; the lanes share k.  Up to some 21000 channels (R = 4: nine blocks of 128 threads an SM) all warps are resident at
// once, and what an SM has more of than others costs nothing, since HBM is the bound and not the SM; beyond that blocks follow as others end
// (28672 x 4096 keeps 5.8 TB/s).
template <typename OUT, int MT, int R>
__global__ void __launch_bounds__(LIN_FEW_THREADS) linear_s8_few_kernel(const LinearParams p) {
    constexpr int U = LIN_FEW_LOADS / R;
    const int lane = threadIdx.x & 31, n0 = (blockIdx.x * (LIN_FEW_THREADS / 32) + (threadIdx.x >> 5)) * R;
    ptx::dependency_wait();
    ptx::dependents_launch();
    if (n0 >= p.N) return;
    int acc[R][MT];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int m = 0; m < MT; ++m) acc[r][m] = 0;
    const int8_t* w[R];
#pragma unroll
    for (int r = 0; r < R; ++r) w[r] = p.w + (long long)(n0 + r < p.N ? n0 + r : n0) * p.ldw;
    for (int k0 = 16 * lane; k0 < p.K; k0 += 512 * U) {
        uint4 b[U][R];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int r = 0; r < R; ++r) b[u][r] = linear_load16(w[r], k0 + 512 * u, p.K, true);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                const uint4 x = linear_load16(p.q + (m < p.M ? m * p.ldq : 0), m < p.M ? k0 + 512 * u : p.K, p.K, false);
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    acc[r][m] = __dp4a((int)b[u][r].x, (int)x.x, acc[r][m]);
                    acc[r][m] = __dp4a((int)b[u][r].y, (int)x.y, acc[r][m]);
                    acc[r][m] = __dp4a((int)b[u][r].z, (int)x.z, acc[r][m]);
                    acc[r][m] = __dp4a((int)b[u][r].w, (int)x.w, acc[r][m]);
                }
            }
    }
    int mine = 0;   // of token lane / R and channel lane % R
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int sum = __reduce_add_sync(0xffffffffu, acc[r][m]);
            if (lane == m * R + r) mine = sum;
        }
    const int m = lane / R, n = n0 + lane % R;
    if (m < MT && m < p.M && n < p.N)
        static_cast<OUT*>(p.y)[m * p.ldy + n] = linear_round<OUT>(fmaf((float)mine * p.s[m], p.ws[n], p.bias ? p.bias[n] : 0.f));
}

// ------------------------------------------------------------------------------------------------ many rows
constexpr int LIN_ROWS = 128;          // of a tile, per CTA
constexpr int LIN_THREADS = 384;
constexpr int LIN_GROUP = 8;           // tiles of rows that are worked through for all channels before the next ones: 2048 rows stay in L2
constexpr uint64_t LIN_WAIT_LIMIT_NS = 200ull * 1000ull * 1000ull;

template <int BN, typename OUT>
struct LinCfg {
    static constexpr int A_BYTES = LIN_ROWS * 128, B_BYTES = BN / 2 * 128, STAGE = A_BYTES + B_BYTES;
    // The epilogue works on units of 128 bytes of 32 rows, which its eight warps, two for each 32 rows of the accumulator, take in turn.
    static constexpr int UNIT = 128 / (int)sizeof(OUT), UNITS = BN / UNIT, WARP_UNITS = (UNITS + 1) / 2, UNIT_BYTES = 32 * 128;
    static constexpr int STAGING = 8 * UNIT_BYTES, WARP_COLS = WARP_UNITS * UNIT, TABLES = 8 * 2 * WARP_COLS * 4;
    static constexpr int BARRIERS = 256, MOST = 227 * 1024 - 1024;
    static constexpr int STAGES = (MOST - STAGING - TABLES - BARRIERS) / STAGE < 8 ? (MOST - STAGING - TABLES - BARRIERS) / STAGE : 8;
    static constexpr int O_STAGING = STAGES * STAGE, O_TABLES = O_STAGING + STAGING, O_BARRIERS = O_TABLES + TABLES;
    static constexpr int SMEM_BYTES = O_BARRIERS + BARRIERS + 1024;   // (the base is moved up to 1024 bytes)
    static constexpr uint32_t ACC_COLS = BN > 128 ? 256 : BN, TMEM_COLS = 2 * ACC_COLS;
    static_assert(STAGES >= 4 && (2 * STAGES + 5) * 8 + 16 <= BARRIERS && BN % 64 == 0 && BN <= 256, "");
};

// One of a pair's two CTAs: what its roles share.
template <int BN, typename OUT>
struct LinBlock {
    using C = LinCfg<BN, OUT>;
    uint32_t base, rank;
    __device__ __forceinline__ uint32_t bar(int i) const { return base + C::O_BARRIERS + 8 * i; }
    __device__ __forceinline__ uint32_t full(int s) const { return bar(s); }                        // (the first CTA's) a stage's loads of both CTAs have landed
    __device__ __forceinline__ uint32_t empty(int s) const { return bar(C::STAGES + s); }           // its MMAs are done
    __device__ __forceinline__ uint32_t acc_full(int a) const { return bar(2 * C::STAGES + a); }    // a tile's MMAs are done
    __device__ __forceinline__ uint32_t acc_empty(int a) const { return bar(2 * C::STAGES + 2 + a); }   // (the first CTA's) both CTAs have read it
    __device__ __forceinline__ uint32_t drain() const { return bar(2 * C::STAGES + 4); }
    __device__ __forceinline__ uint32_t flags() const { return bar(2 * C::STAGES + 5); }            // abort, skip, tensor-memory address
    __device__ __forceinline__ bool wait(uint32_t b, uint32_t parity) const { return ptx::mbar_wait_warp_s(b, parity, flags(), LIN_WAIT_LIMIT_NS); }
};

__device__ __forceinline__ void linear_tile(const LinearParams& p, int tile, int& tm, int& tn) {
    const int per = LIN_GROUP * p.tiles_n, first = tile / per * LIN_GROUP, rest = tile % per;
    const int rows = p.tiles_m - first < LIN_GROUP ? p.tiles_m - first : LIN_GROUP;
    tm = first + rest % rows;
    tn = rest / rows;
}

template <int BN, typename OUT>
__device__ __forceinline__ void linear_load(const LinearParams& p, const LinBlock<BN, OUT>& k, const CUtensorMap& ma, const CUtensorMap& mb, int pair, int pairs) {
    using C = LinCfg<BN, OUT>;
    const int tiles = p.tiles_m * p.tiles_n, kblocks = (p.K + 127) / 128;
    const uint32_t el = ptx::elect_one();
    int s = 0;
    uint32_t phase = 1;   // the first pass finds every stage empty
    for (int tile = pair; tile < tiles; tile += pairs) {
        int tm, tn;
        linear_tile(p, tile, tm, tn);
        const int row_a = tm * 2 * LIN_ROWS + (int)k.rank * LIN_ROWS, row_b = tn * BN + (int)k.rank * (BN / 2);
        for (int kb = 0; kb < kblocks; ++kb) {
            if (!k.wait(k.empty(s), phase)) {
                // loads of this warp may be in flight: they land within microseconds, the block leaves after two milliseconds
                for (const uint64_t t0 = ptx::globaltimer_ns(); ptx::globaltimer_ns() - t0 < ptx::DRAIN_LIMIT_NS;) __nanosleep(1000);
                return;
            }
            if (el) {
                const uint32_t full = ptx::cluster_address(k.full(s), 0), to = k.base + s * C::STAGE;
                if (k.rank == 0) ptx::mbar_arrive_expect_tx(k.full(s), 2 * C::STAGE);
                ptx::tma_load_2d_pair(to, &ma, full, kb * 128, row_a);
                ptx::tma_load_2d_pair(to + C::A_BYTES, &mb, full, kb * 128, row_b);
            }
            __syncwarp();
            if (++s == C::STAGES) { s = 0; phase ^= 1; }
        }
    }
    // every arrival that the MMAs still owe this CTA has come in before it leaves
    for (int i = 0; i < C::STAGES; ++i) {
        if (!k.wait(k.empty(s), phase)) return;
        if (++s == C::STAGES) { s = 0; phase ^= 1; }
    }
}

template <int BN, typename OUT>
__device__ __forceinline__ void linear_issue(const LinearParams& p, const LinBlock<BN, OUT>& k, uint32_t tmem, int pair, int pairs) {
    using C = LinCfg<BN, OUT>;
    constexpr uint32_t IDESC = ptx::idesc_s8_s32(2 * LIN_ROWS, BN), HI = ptx::desc_hi_sw128(1024);
    const int tiles = p.tiles_m * p.tiles_n, kblocks = (p.K + 127) / 128;
    const uint32_t el = ptx::elect_one();
    int s = 0, n = 0;
    uint32_t phase = 0;
    bool ok = true;
    for (int tile = pair; tile < tiles && ok; tile += pairs, ++n) {
        const int acc = n & 1;
        ok = k.wait(k.acc_empty(acc), ((n >> 1) & 1) ^ 1);
        ptx::tc_fence_after_sync();
        const uint32_t d = tmem + acc * C::ACC_COLS;
        for (int kb = 0; kb < kblocks && ok; ++kb) {
            ok = k.wait(k.full(s), phase);
            if (!ok) break;
            ptx::tc_fence_after_sync();
            const uint32_t a = ptx::desc_lo(k.base + s * C::STAGE, 16), b = ptx::desc_lo(k.base + s * C::STAGE + C::A_BYTES, 16);
            const int steps = p.K - kb * 128 > 96 ? 4 : (p.K - kb * 128 + 31) / 32;   // (behind K there are zeros)
            for (int i = 0; i < steps; ++i) ptx::mma_s8_pair(el, d, a + 2 * i, b + 2 * i, HI, IDESC, kb + i > 0);
            ptx::mma_commit_pair(el, k.empty(s));
            if (++s == C::STAGES) { s = 0; phase ^= 1; }
        }
        if (ok) ptx::mma_commit_pair(el, k.acc_full(acc));
    }
    if (!ok) {   // the MMAs in flight end before the tensor memory is freed
        ptx::mma_commit_pair(el, k.drain());
        ptx::mbar_wait_drain(k.drain(), 0, ptx::DRAIN_LIMIT_NS);
    }
}

template <int BN, typename OUT>
__device__ __forceinline__ void linear_store(const LinearParams& p, const LinBlock<BN, OUT>& k, const CUtensorMap& my, uint32_t tmem, int pair, int pairs) {
    using C = LinCfg<BN, OUT>;
    constexpr int PER16 = 16 / (int)sizeof(OUT), COLS = (C::WARP_COLS + 31) / 32;
    const int tiles = p.tiles_m * p.tiles_n, lane = threadIdx.x & 31, warp = threadIdx.x / 32 - 4, quad = warp & 3, side = warp >> 2;
    const uint32_t to = k.base + C::O_STAGING + warp * C::UNIT_BYTES, table = k.base + C::O_TABLES + warp * 2 * C::WARP_COLS * 4;
    const uint32_t acc_empty = ptx::cluster_address(k.acc_empty(0), 0);
    // A tile's scales: the lane's row's, and those and the biases of the columns of the warp's units (unit 2 j + its turn), a lane's
    // share of them.  They are loaded a tile ahead and handed out through a table of the warp's own.
    float sm, wsc[COLS], bia[COLS];
    auto fetch = [&](int tile, int n) {
        if (tile >= tiles) return;
        int tm, tn;
        linear_tile(p, tile, tm, tn);
        const long long m = (long long)tm * 2 * LIN_ROWS + k.rank * LIN_ROWS + quad * 32 + lane;
        sm = m < p.M ? p.s[m] : 0.f;
#pragma unroll
        for (int j = 0; j < COLS; ++j) {
            const int at = 32 * j + lane, unit = 2 * (at / C::UNIT) + ((side + n) & 1), col = tn * BN + unit * C::UNIT + at % C::UNIT;
            const bool in = unit < C::UNITS && col < p.N;
            wsc[j] = in ? p.ws[col] : 0.f;
            bia[j] = in && p.bias ? p.bias[col] : 0.f;
        }
    };
    fetch(pair, 0);
    int n = 0;
    for (int tile = pair; tile < tiles; tile += pairs, ++n) {
        int tm, tn;
        linear_tile(p, tile, tm, tn);
        const int acc = n & 1, turn = (side + n) & 1;
        const long long row0 = (long long)tm * 2 * LIN_ROWS + k.rank * LIN_ROWS + quad * 32;
        const float s_row = sm;
        __syncwarp();   // the tile before is done with the table
#pragma unroll
        for (int j = 0; j < COLS; ++j) {
            asm volatile("st.shared.f32 [%0], %1;" ::"r"(table + 4 * (32 * j + lane)), "f"(wsc[j]) : "memory");
            asm volatile("st.shared.f32 [%0], %1;" ::"r"(table + 4 * (C::WARP_COLS + 32 * j + lane)), "f"(bia[j]) : "memory");
        }
        __syncwarp();
        fetch(tile + pairs, n + 1);
        if (!k.wait(k.acc_full(acc), (n >> 1) & 1)) break;
        ptx::tc_fence_after_sync();
        const uint32_t from = tmem + ((uint32_t)(quad * 32) << 16) + acc * C::ACC_COLS;
        const uint64_t s2 = ptx::pack2(s_row, s_row);
#pragma unroll 1
        for (int j = 0, u = turn; j < C::WARP_UNITS; ++j, u += 2) {
            const bool there = u < C::UNITS, last = u + 2 >= C::UNITS;
            uint32_t r[C::UNIT];
            if (there) {
#pragma unroll
                for (int c = 0; c < C::UNIT; c += 32) ptx::tmem_ld32(from + u * C::UNIT + c, r + c);
                ptx::tmem_wait_ld();
            }
            if (last) {   // the accumulator may be filled again
                ptx::tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive_cluster(acc_empty + 8 * acc);
            }
            if (!there) break;
            if (lane == 0) ptx::bulk_wait_read();   // the store before is done with the staged unit
            __syncwarp();
#pragma unroll
            for (int i = 0; i < 8; ++i) {   // pieces of 16 bytes
                uint64_t v[PER16 / 2];
#pragma unroll
                for (int e = 0; e < PER16; e += 4) {
                    const uint32_t at = table + 4 * (j * C::UNIT + i * PER16 + e);
                    uint64_t a[2], b[2];
                    asm volatile("ld.shared.v2.b64 {%0,%1}, [%2];" : "=l"(a[0]), "=l"(a[1]) : "r"(at));
                    asm volatile("ld.shared.v2.b64 {%0,%1}, [%2];" : "=l"(b[0]), "=l"(b[1]) : "r"(at + 4 * C::WARP_COLS));
                    const uint32_t* q = r + i * PER16 + e;
                    v[e / 2] = ptx::fma2(ptx::mul2(ptx::pack2((float)(int)q[0], (float)(int)q[1]), s2), a[0], b[0]);
                    v[e / 2 + 1] = ptx::fma2(ptx::mul2(ptx::pack2((float)(int)q[2], (float)(int)q[3]), s2), a[1], b[1]);
                }
                uint32_t w[4];
#pragma unroll
                for (int e = 0; e < PER16 / 2; ++e) {
                    float lo, hi;
                    ptx::unpack2(v[e], lo, hi);
                    if constexpr (sizeof(OUT) == 2) w[e] = ptx::pack_bf16(lo, hi);
                    else { w[2 * e] = __float_as_uint(lo); w[2 * e + 1] = __float_as_uint(hi); }
                }
                // rows of 128 bytes with the swizzle of the tensor map: free of bank conflicts, and what the store expects
                ptx::st_shared_v4(to + lane * 128 + ((i ^ (lane & 7)) << 4), w[0], w[1], w[2], w[3]);
            }
            const int col0 = tn * BN + u * C::UNIT;
            if (col0 + C::UNIT <= p.tma_cols) {
                ptx::fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) {
                    if (row0 < p.M && col0 < p.N) ptx::tma_store_2d(&my, to, col0, (int)row0);
                    ptx::bulk_commit();
                }
            } else {   // rows that do not begin or end on 16 bytes: a warp stores one row after the other, 4 bytes a lane if they begin on 4
                __syncwarp();
                const long long rows = p.M - row0;
                const int cols = p.N - col0;
                OUT* dst = static_cast<OUT*>(p.y) + row0 * p.ldy + col0;
                auto staged = [&](int i, int c) { return to + i * 128 + (((c / PER16) ^ (i & 7)) << 4) + c % PER16 * (int)sizeof(OUT); };
                if (sizeof(OUT) == 4 || ((reinterpret_cast<uintptr_t>(p.y) | (uintptr_t)(p.ldy * 2)) & 3) == 0) {
                    constexpr int E = 4 / (int)sizeof(OUT);   // elements of 4 bytes
#pragma unroll 8
                    for (int i = 0; i < 32; ++i) {
                        uint32_t v;
                        asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(staged(i, E * lane)));
                        OUT* at = dst + i * p.ldy + E * lane;
                        if (i < rows && E * lane + E <= cols) *reinterpret_cast<uint32_t*>(at) = v;
                        else if (i < rows && E * lane < cols) *reinterpret_cast<unsigned short*>(at) = (unsigned short)v;   // (a last odd column)
                    }
                } else {
#pragma unroll 8
                    for (int i = 0; i < 32; ++i) {
                        unsigned short v[2];
#pragma unroll
                        for (int h = 0; h < 2; ++h) asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v[h]) : "r"(staged(i, lane + 32 * h)));
#pragma unroll
                        for (int h = 0; h < 2; ++h)
                            if (i < rows && lane + 32 * h < cols) *reinterpret_cast<unsigned short*>(dst + i * p.ldy + lane + 32 * h) = v[h];
                    }
                }
                __syncwarp();
            }
            if (last) break;
        }
    }
    if (lane == 0) ptx::bulk_wait_all();
}

template <int BN, typename OUT>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(LIN_THREADS, 1)
linear_s8_kernel(const __grid_constant__ CUtensorMap ma, const __grid_constant__ CUtensorMap mb, const __grid_constant__ CUtensorMap my, const LinearParams p) {
    using C = LinCfg<BN, OUT>;
    extern __shared__ uint8_t smem[];
    LinBlock<BN, OUT> k;
    k.base = (ptx::smem_u32(smem) + 1023u) & ~1023u;
    k.rank = ptx::cluster_rank();
    const int warp = threadIdx.x >> 5, pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    volatile int* flags = static_cast<volatile int*>(__cvta_shared_to_generic(k.flags()));
    if (threadIdx.x == 0) {
        for (int s = 0; s < C::STAGES; ++s) { ptx::mbar_init(k.full(s), 1); ptx::mbar_init(k.empty(s), 1); }
        for (int a = 0; a < 2; ++a) { ptx::mbar_init(k.acc_full(a), 1); ptx::mbar_init(k.acc_empty(a), 2 * 8); }
        ptx::mbar_init(k.drain(), 1);
        flags[0] = 0;
        ptx::fence_mbar_init();
    }
    if (warp == 2) ptx::tmem_alloc_pair(k.flags() + 8, C::TMEM_COLS);
    ptx::dependency_wait();
    ptx::dependents_launch();
    if (threadIdx.x == 0) flags[1] = *reinterpret_cast<volatile int*>(p.status);   // an earlier kernel timed out: both CTAs do nothing if either sees it
    __syncwarp();
    ptx::tc_fence_before_sync();
    ptx::cluster_sync();
    ptx::tc_fence_after_sync();
    const bool skip = ptx::ld_cluster(ptx::cluster_address(k.flags() + 4, 0)) | ptx::ld_cluster(ptx::cluster_address(k.flags() + 4, 1));
    const uint32_t tmem = flags[2];
    if (!skip) {
        if (warp == 0) linear_load<BN, OUT>(p, k, ma, mb, pair, pairs);
        else if (warp == 1 && k.rank == 0) linear_issue<BN, OUT>(p, k, tmem, pair, pairs);
        else if (warp >= 4) linear_store<BN, OUT>(p, k, my, tmem, pair, pairs);
    }
    __syncwarp();
    ptx::tc_fence_before_sync();
    ptx::cluster_sync();   // neither CTA leaves, or frees its tensor memory, while the other one may still reach into it
    ptx::tc_fence_after_sync();
    if (warp == 2) ptx::tmem_dealloc_pair(tmem, C::TMEM_COLS);
    if (threadIdx.x == 0 && flags[0]) atomicExch(p.status, 1);
}

// ------------------------------------------------------------------------------------------------ some rows
// Up to 256 rows: the weights stream past the tokens, so they are the operand with 128 rows (channels), the tokens the one with NT columns,
// and the cluster's CTAs share k.  When all are done, each writes its partial sums, integers, of a token into the shared memory of the
// CTA that adds them up (writes do not wait for one another; fetched by reads, 64 tokens took 4 us more).  Tiles of up to 64 tokens have three
// CTAs an SM: what it has in flight is 150 KB and more.
constexpr int LIN_THIN_THREADS = 192;

template <int NT>
struct ThinCfg {
    static constexpr int W_BYTES = 128 * 128, Q_BYTES = NT * 128, STAGE = W_BYTES + Q_BYTES;
    static constexpr int STAGES = NT <= 16 ? 4 : NT <= 128 ? 3 : 4, RESIDENT = NT <= 64 ? 3 : NT <= 128 ? 2 : 1;
    static constexpr int O_BARRIERS = STAGES * STAGE, SMEM_BYTES = O_BARRIERS + 128 + 1024;
    static constexpr uint32_t TMEM_COLS = NT < 32 ? 32 : NT;
    // (NT / 4 + 7) / parts groups of four tokens and 128 channels from each of up to 8 CTAs
    static_assert((NT / 4 + 7) * 2048 <= STAGES * STAGE && (2 * STAGES + 2) * 8 + 16 <= 128 && RESIDENT * (SMEM_BYTES + 1024) <= 228 * 1024, "");
};

template <int NT, typename OUT>
__global__ void __launch_bounds__(LIN_THIN_THREADS)
linear_s8_thin_kernel(const __grid_constant__ CUtensorMap mw, const __grid_constant__ CUtensorMap mq, const LinearParams p) {
    using C = ThinCfg<NT>;
    extern __shared__ uint8_t smem[];
    const uint32_t base = (ptx::smem_u32(smem) + 1023u) & ~1023u, bars = base + C::O_BARRIERS;
    auto full = [&](int s) { return bars + 8 * s; };
    auto empty = [&](int s) { return bars + 8 * (C::STAGES + s); };
    const uint32_t done = bars + 8 * (2 * C::STAGES), drain = done + 8, flag_addr = done + 16;
    volatile int* flags = static_cast<volatile int*>(__cvta_shared_to_generic(flag_addr));   // abort, skip, tensor-memory address
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, parts = p.ksplit;
    const int part = parts > 1 ? (int)ptx::cluster_rank() : 0, tile = blockIdx.x / parts;
    const int kblocks = (p.K + 127) / 128, first = (int)((long long)kblocks * part / parts), last = (int)((long long)kblocks * (part + 1) / parts);
    if (threadIdx.x == 0) {
        for (int s = 0; s < C::STAGES; ++s) { ptx::mbar_init(full(s), 1); ptx::mbar_init(empty(s), 1); }
        ptx::mbar_init(done, 1);
        ptx::mbar_init(drain, 1);
        flags[0] = 0;
        ptx::fence_mbar_init();
    }
    if (warp == 1) { ptx::tmem_alloc(flag_addr + 8, C::TMEM_COLS); ptx::tmem_relinquish(); }
    ptx::dependency_wait();
    ptx::dependents_launch();
    if (threadIdx.x == 0) flags[1] = *reinterpret_cast<volatile int*>(p.status);   // an earlier kernel timed out: nothing is computed
    ptx::tc_fence_before_sync();
    __syncthreads();
    ptx::tc_fence_after_sync();
    const uint32_t tmem = flags[2];
    const bool skip = flags[1];
    if (skip) {
    } else if (warp == 0) {
        const uint32_t el = ptx::elect_one();
        int s = 0;
        uint32_t phase = 1;
        bool ok = true;
        for (int kb = first; kb < last && ok; ++kb) {
            ok = ptx::mbar_wait_warp_s(empty(s), phase, flag_addr, LIN_WAIT_LIMIT_NS);
            if (ok && el) {
                ptx::mbar_arrive_expect_tx(full(s), C::STAGE);
                ptx::tma_load_2d(base + s * C::STAGE, &mw, full(s), kb * 128, tile * 128);
                ptx::tma_load_2d(base + s * C::STAGE + C::W_BYTES, &mq, full(s), kb * 128, 0);
            }
            __syncwarp();
            if (++s == C::STAGES) { s = 0; phase ^= 1; }
        }
        if (!ok)   // loads in flight land within microseconds, the block leaves after two milliseconds
            for (const uint64_t t0 = ptx::globaltimer_ns(); ptx::globaltimer_ns() - t0 < ptx::DRAIN_LIMIT_NS;) __nanosleep(1000);
    } else if (warp == 1) {
        constexpr uint32_t IDESC = ptx::idesc_s8_s32(128, NT), HI = ptx::desc_hi_sw128(1024);
        const uint32_t el = ptx::elect_one();
        int s = 0;
        uint32_t phase = 0;
        bool ok = true;
        for (int kb = first; kb < last; ++kb) {
            ok = ptx::mbar_wait_warp_s(full(s), phase, flag_addr, LIN_WAIT_LIMIT_NS);
            if (!ok) break;
            ptx::tc_fence_after_sync();
            const uint32_t a = ptx::desc_lo(base + s * C::STAGE, 16), b = ptx::desc_lo(base + s * C::STAGE + C::W_BYTES, 16);
            const int steps = p.K - kb * 128 > 96 ? 4 : (p.K - kb * 128 + 31) / 32;   // (behind K there are zeros)
            for (int i = 0; i < steps; ++i) ptx::mma_s8(el, tmem, a + 2 * i, b + 2 * i, HI, IDESC, kb > first || i > 0);
            ptx::mma_commit_p(el, empty(s));
            if (++s == C::STAGES) { s = 0; phase ^= 1; }
        }
        if (ok) ptx::mma_commit_p(el, done);
        else {   // the MMAs in flight end before the tensor memory is freed
            ptx::mma_commit_p(el, drain);
            ptx::mbar_wait_drain(drain, 0, ptx::DRAIN_LIMIT_NS);
        }
    }
    const int quad = warp & 3, channel = quad * 32 + lane, n = tile * 128 + channel;
    bool ok = !skip && warp >= 2 && ptx::mbar_wait_warp_s(done, 0, flag_addr, LIN_WAIT_LIMIT_NS);
    if (ok) ptx::tc_fence_after_sync();
    const bool in = ok && n < p.N;
    const float wsc = in ? p.ws[n] : 0.f, bias = in && p.bias ? p.bias[n] : 0.f;
    auto store = [&](int m, int sum, float sm) { static_cast<OUT*>(p.y)[m * p.ldy + n] = linear_round<OUT>(fmaf((float)sum * sm, wsc, bias)); };
    // Each CTA adds up the same number of tokens, four by four: the sums of four tokens and a channel are 16 bytes of each CTA's.
    const int quads = ((p.M + 3) / 4 + parts - 1) / parts;
    __syncwarp();
    if (parts > 1) ptx::cluster_sync();   // all loads have landed, all MMAs have read them: the rings' memory is free
    if (ok) {
        int to = 0, slot = 0;
#pragma unroll 1
        for (int c = 0; c < NT && c < p.M; c += 16) {
            uint32_t r[16];
            ptx::tmem_ld16(tmem + ((uint32_t)(quad * 32) << 16) + c, r);
            ptx::tmem_wait_ld();
#pragma unroll
            for (int j = 0; j < 16; j += 4) {
                if (parts > 1) {
                    if (to < parts) ptx::st_cluster_v4(ptx::cluster_address(base + ((part * quads + slot) * 128 + channel) * 16, to), r[j], r[j + 1], r[j + 2], r[j + 3]);
                    if (++slot == quads) { slot = 0; ++to; }
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (c + j + e < p.M && in) store(c + j + e, (int)r[j + e], p.s[c + j + e]);
                }
            }
        }
    }
    __syncwarp();
    ptx::tc_fence_before_sync();
    if (parts > 1) {
        ptx::cluster_sync();
        const int4* sums = static_cast<const int4*>(__cvta_shared_to_generic(base)) + channel;
        const int m0 = part * quads * 4;   // the first of this CTA's tokens
        for (int i0 = 0; i0 < quads && m0 + 4 * i0 < p.M; i0 += 8) {
            // the scales of the next 32 tokens, a lane each
            const float sv = m0 + 4 * i0 + lane < p.M ? p.s[m0 + 4 * i0 + lane] : 0.f;
#pragma unroll 2
            for (int i = 0; i < 8; ++i) {
                if (i0 + i >= quads) break;
                int4 sum = make_int4(0, 0, 0, 0);
#pragma unroll
                for (int r = 0; r < 8; ++r) {
                    const int4 v = r < parts ? sums[(r * quads + i0 + i) * 128] : make_int4(0, 0, 0, 0);
                    sum.x += v.x; sum.y += v.y; sum.z += v.z; sum.w += v.w;
                }
                const int m = m0 + 4 * (i0 + i), all[4] = {sum.x, sum.y, sum.z, sum.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float sm = __shfl_sync(0xffffffffu, sv, 4 * i + e);
                    if (in && m + e < p.M) store(m + e, all[e], sm);
                }
            }
        }
    }
    __syncthreads();
    ptx::tc_fence_after_sync();
    if (warp == 1) ptx::tmem_dealloc(tmem, C::TMEM_COLS);
    if (threadIdx.x == 0 && flags[0]) atomicExch(p.status, 1);
}

}  // namespace tvm_attn

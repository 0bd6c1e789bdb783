// RMSNorm over the model width with the residual's addition and a tangent, its backward through all outputs, and its
// 8-bit form: the norm in front of the attention of the paper's transformer (Sec. 4 "semi-Lipschitz control": LayerNorm
// replaced by RMSNorm without a learnable scale; App. "Lipschitzness of RMSNorm" for the Jacobian).  Per row of D elements:
//     h = x + res     r = sqrt(mean(h^2) + eps)     u = h / r     y = g u
//     th = tx + tres                                ty = g J th   with J v = (v - u (u . v) / D) / r
// Streaming work, every tensor read or written once, bound by HBM once enough bytes are in flight.  A row has a 16-byte chunk on
// each of P lanes of a warp, or 1, 2 or 4 chunks on each thread of a block of its own, and stays in registers between its loads
// and its stores: few registers a thread, so that the blocks of an SM, each a row further on, cover for one another.  The sums over a
// row, the dot products and the scale's gradient are fp32.  The norm is that of the sum before it is rounded to the type that h is
// stored in.  Measured on B200, (16384, 1152) bf16, outputs given: norm with residual and tangents 50 us (302 MB, 6.0 TB/s of 6.5), without
// tangents 26.9, backward with residual, tangents and scale 54.5 (5.5 TB/s), without tangents 29.3, 8-bit rows 27.0, without a norm 20.1.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "chunks.cuh"
#include "sm100_ptx.cuh"

namespace tvm_attn {

// The rows of a (B, T, D) tensor, strides in bytes.
struct RowsPtr {
    char* p;
    long long row, batch;
};

struct RowNormParams {
    RowsPtr in[6];    // forward: x, res, tx, tres; backward: h, dy, dh, th, dty, dth
    RowsPtr out[4];   // forward: y (or the 8-bit rows), h, ty, th; backward: dx, dtx
    const float* g;   // null: no learnable scale
    float* aux;       // 8-bit rows: their scales; backward: partial sums of the scale's gradient, or null
    unsigned total, T;
    int D, P;         // P: lanes of a row (all threads of the block where a row has one of its own)
    float eps;
    bool flat;        // every tensor is one dimension of rows less than 4 GB apart
    bool same;        // and all have the same stride and less than 4 GB
    bool norm;        // 8-bit rows: of the norm's output (else of x + res itself)
};

constexpr int ROWNORM_THREADS = 256;   // of a block whose rows are on warps
// Chunks of a row with one on each thread, at most: two a thread from there on.  The backward sets it (the norms differ by 5 % at most between 96 and 256): with
// tangents and 38 MB a tensor of bf16 rows, 1152 wide 53.9 us as it is, 63.8 with two chunks a thread (a limit of 128); 1408 wide 58.6 as it is and 55.9 with one
// (a limit of 192), but then all blocks are compiled for 192 threads and fewer registers each, and 1152 wide takes 58.1, 512 wide 90.8 instead of 81.2.
constexpr int ROWNORM_SINGLE = 160;
// Threads that a block with one row can have, C chunks each.
template <typename T, int C> constexpr int rownorm_block_threads() { return C == 4 && sizeof(T) == 4 ? 1024 : C == 1 ? ROWNORM_SINGLE : 512; }
// Blocks of the backward on an SM: as many as the registers let in (a block walks over its rows from the start to the end of the
// launch, so one that waits for another's end would double the time), of one chunk a thread those of ROWNORM_SINGLE threads, whatever their own
// number: narrower ones leave registers unused (512 wide with tangents 81 us where 1152 take 54).  `threads`: of a block with one row of C chunks a
// thread, 0 for rows on warps.
__host__ __device__ constexpr int rownorm_bwd_resident(int threads, int C, bool tan) {
    return threads == 0 ? (tan ? 2 : 4) : C == 1 ? (tan ? 4 : 7) : threads <= 512 ? 512 / threads : 1;
}
// All of them.  A fixed number: the partial sums of the scale's gradient, a row per block, have a size and an order that do not
// depend on the device.
__host__ __device__ constexpr int rownorm_bwd_blocks(int threads, int C, bool tan) { return 148 * rownorm_bwd_resident(threads, C, tan); }

// `base` moved on by `row` rows of tensor t: one instruction where the rows are one dimension.
__device__ __forceinline__ char* row_of(char* base, const RowsPtr& t, unsigned row, const RowNormParams& p) {
    if (p.flat) return base + (size_t)row * (unsigned)t.row;
    const unsigned b = row / p.T;
    return base + (size_t)b * (size_t)t.batch + (size_t)(row - b * p.T) * (size_t)t.row;
}

// The lanes of one row and their columns.  VEC: a chunk is 16 contiguous bytes.  Otherwise (a pointer, stride or width that is
// no multiple of 16 bytes) the elements of a chunk are P apart, so that an instruction still touches contiguous bytes.
template <typename T, bool VEC>
struct RowLane {
    static constexpr int V = RmsVec<T>::N;
    int c, P, D;
    __device__ __forceinline__ int col(int i, int e) const { return VEC ? (c + P * i) * V + e : c + P * (i * V + e); }
    // A chunk as it lies in memory, zeros behind the row.  `row`: its address at column col(0, 0).
    __device__ __forceinline__ uint4 raw(const T* row, bool act, int i) const {
        uint4 q = make_uint4(0, 0, 0, 0);
        if constexpr (VEC) {
            if (act && col(i, 0) < D) q = *reinterpret_cast<const uint4*>(row + P * i * V);
        } else {
            uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (act && col(i, e) < D) {
                    const T x = row[P * (i * V + e)];
                    if constexpr (V == 4) w[e] = __float_as_uint(x);
                    else w[e / 2] |= (uint32_t)__bfloat16_as_ushort(x) << (16 * (e & 1));
                }
            q = make_uint4(w[0], w[1], w[2], w[3]);
        }
        return q;
    }
    __device__ __forceinline__ void store(T* row, int i, const uint64_t (&v)[V / 2]) const {
        if constexpr (VEC) {
            if (col(i, 0) < D) rms_store(row + P * i * V, v);
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e) {
                float a, b;
                ptx::unpack2(v[e / 2], a, b);
                if (col(i, e) < D) row[P * (i * V + e)] = (T)(e & 1 ? b : a);
            }
        }
    }
    // The scale's elements for a chunk: 1 where there is no scale, 0 behind the row.
    __device__ __forceinline__ void scale(const float* g, int i, uint64_t (&v)[V / 2]) const {
        if (VEC && g) {   // (the scale is aligned too, and whole chunks stand in a row or behind it)
#pragma unroll
            for (int e = 0; e < V / 2; e += 2) {
                float4 q = make_float4(0.f, 0.f, 0.f, 0.f);
                if (col(i, 0) < D) q = *reinterpret_cast<const float4*>(g + col(i, 2 * e));
                v[e] = ptx::pack2(q.x, q.y);
                v[e + 1] = ptx::pack2(q.z, q.w);
            }
            return;
        }
#pragma unroll
        for (int e = 0; e < V; e += 2) {
            float a = 1.f, b = 1.f;
            if (g) {
                a = col(i, e) < D ? g[col(i, e)] : 0.f;
                b = col(i, e + 1) < D ? g[col(i, e + 1)] : 0.f;
            }
            v[e / 2] = ptx::pack2(a, b);
        }
    }
    // Address of row `row` of a tensor of T at the lane's first column.  SAME: all tensors share one 32-bit offset, and nothing but that
    // is held for them ((16384, 1152) bf16: backward 60.8 -> 57.3 us; the forward with tangents 49.7 -> 58.3, so it has its own for each).
    template <bool SAME>
    __device__ __forceinline__ T* at(const RowsPtr& t, unsigned row, const RowNormParams& p) const {
        if (SAME) return reinterpret_cast<T*>(t.p + (row * (unsigned)p.in[0].row + (unsigned)(col(0, 0) * (int)sizeof(T))));
        return reinterpret_cast<T*>(row_of(t.p + col(0, 0) * (int)sizeof(T), t, row, p));
    }
};

// Asks for row `row` of the N tensors, which a block takes next: a whole row by one instruction, so that its loads find it in L2.
// (16384, 1152) bf16: backward 9 % faster, without tangents 16 %, 8 bits 8 %, norm of a sum 2 %; not with tangents in the forward, which has
// its bytes in flight (14 % slower), nor for rows on warps ((131072, 128): 4 % slower).  A row ahead in registers instead: 3 % faster for the
// norm of a sum, 9 % slower with tangents.
template <int N>
__device__ __forceinline__ void row_prefetch(const RowNormParams& p, unsigned row, int bytes) {   // a thread for each tensor
    if (threadIdx.x < N && row < p.total) {
        const RowsPtr& t = p.in[threadIdx.x];
        if (t.p) ptx::prefetch_l2(row_of(t.p, t, row, p), (uint32_t)bytes);
    }
}

__device__ __forceinline__ float max_nan(float a, float b) {   // a NaN on either side stays
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// The sums of N values (the last one a maximum with MAX, where N = 2) over P lanes, each on some of them: the lanes halve the
// values among them with every step.  5 values: by the three highest bits of the lane's place, 000, 001, 010, 100 and 101 hold values
// 0 to 4, the others nothing; 2 values: by the highest bit.
template <int N, bool MAX>
__device__ __forceinline__ float row_scatter(const float (&v)[N], int P, int lane) {
    float part[N];
#pragma unroll
    for (int k = 0; k < N; ++k) part[k] = v[k];
    int off = P >> 1, n = N;
    const bool last = lane & off;
#pragma unroll
    for (int step = 0; step < 3; ++step) {   // 5 -> 3 -> 2 -> 1
        if (n == 1) break;
        const bool high = lane & off;
        const int half = (n + 1) / 2;
#pragma unroll
        for (int k = 0; k < (N + 1) / 2; ++k) {
            if (k >= half) continue;
            const float lo = part[k], hi = k + half < n ? part[k + half < N ? k + half : 0] : 0.f;
            const float keep = high ? hi : lo, w = __shfl_xor_sync(0xffffffffu, high ? lo : hi, off);
            part[k] = MAX && high ? max_nan(keep, w) : keep + w;
        }
        n = half;
        off >>= 1;
    }
    for (; off > 0; off >>= 1) {
        const float w = __shfl_xor_sync(0xffffffffu, part[0], off);
        part[0] = MAX && last ? max_nan(part[0], w) : part[0] + w;
    }
    return part[0];
}
// The same, all sums on all lanes, the same bits on each.
template <int N, bool MAX>
__device__ __forceinline__ void row_all(float (&v)[N], int P, int lane) {
    if (N == 1 || P < 8) {
        for (int off = P >> 1; off > 0; off >>= 1)
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const float w = __shfl_xor_sync(0xffffffffu, v[k], off);
                v[k] = MAX && k == N - 1 ? max_nan(v[k], w) : v[k] + w;
            }
        return;
    }
    const float part = row_scatter<N, MAX>(v, P, lane);
    const int first = lane & ~(P - 1), bit = N == 2 ? P >> 1 : P >> 3;
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = __shfl_sync(0xffffffffu, part, first + (k < 3 ? k : k + 1) * bit);
}
// The same for a row of a warp's lanes or, with BLOCK, of all threads of a block: `slot`, 32 N floats of shared memory, zeros behind
// the block's warps.  Two slots are used in turn, so that one barrier a reduction is enough.
template <int N, bool MAX, bool BLOCK>
__device__ __forceinline__ void row_reduce(float (&v)[N], int P, float* slot) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if constexpr (!BLOCK) {
        row_all<N, MAX>(v, P, lane);
    } else {
        const float part = row_scatter<N, MAX>(v, 32, lane);
        const int place = lane >> (N == 1 ? 5 : N == 2 ? 4 : 2), id = N == 5 && place > 2 ? place - 1 : place;
        if ((lane & (N == 1 ? 31 : N == 2 ? 15 : 3)) == 0 && (N < 5 || (place != 3 && place < 6))) slot[32 * id + warp] = part;
        __syncthreads();
        if (blockDim.x <= 256) {   // the parts of up to 8 warps, by every thread
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const float4 q = *reinterpret_cast<const float4*>(slot + 32 * k);
                v[k] = MAX && k == N - 1 ? max_nan(max_nan(q.x, q.y), max_nan(q.z, q.w)) : (q.x + q.y) + (q.z + q.w);
            }
            if (blockDim.x > 128)
#pragma unroll
                for (int k = 0; k < N; ++k) {
                    const float4 q = *reinterpret_cast<const float4*>(slot + 32 * k + 4);
                    v[k] = MAX && k == N - 1 ? max_nan(v[k], max_nan(max_nan(q.x, q.y), max_nan(q.z, q.w))) : v[k] + ((q.x + q.y) + (q.z + q.w));
                }
        } else {
#pragma unroll
            for (int k = 0; k < N; ++k) v[k] = slot[32 * k + lane];   // (a maximum is one of magnitudes)
            row_all<N, MAX>(v, 32, lane);
        }
    }
}
// Zeros in the slots, for all threads of the block.
__device__ __forceinline__ void clear_slots(float* slots, int n) {
    for (int i = threadIdx.x; i < n; i += blockDim.x) slots[i] = 0.f;
    __syncthreads();
}

// Rows whose sum of squares leaves the range of fp32, or comes near its ends, are summed again with their elements multiplied by a power of
// two.  (With eps of ordinary size a row of tiny elements needs none.)  The first factor brings every such sum into the range (the largest
// element, 2^42 to 2^128 or 2^-149 to 2^-49, to 2^-54 to 2^47); the second one, from what the first sum says, makes r about 2^aim.
__device__ __forceinline__ bool row_leaves(float ss, float eps) { return !(ss <= 1e30f) || (ss < 1e-30f && eps < 1e-30f); }
__device__ __forceinline__ float row_first(float ss) { return ss < 1e-30f ? 0x1p96f : 0x1p-96f; }
// `ms`: r^2 of elements multiplied by `first`.  1 where there is nothing to be brought back: a row of zeros, an infinity or a NaN.
__device__ __forceinline__ float row_power(float first, float ms, int aim) {
    if (!(ms > 0.f && ms <= 3.4028235e38f)) return 1.f;
    const int n = (first < 1.f ? -96 : 96) + aim - (((int)(__float_as_uint(ms) >> 23) - 127) >> 1);   // -144 to 127
    return __uint_as_float(n >= 127 ? 254u << 23 : n >= -126 ? (uint32_t)(n + 127) << 23 : 1u << (n + 149));
}

// ROW_NORM: y (h, ty, th).  ROW_NORM_TAN: with tangents.  ROW_S8: 8-bit rows q = rint(v / s), s = max|v| / 127, of v = y or x + res;
// a row that holds an infinity or a NaN gets a scale that is not finite, and zeros.
enum { ROW_NORM = 0, ROW_NORM_TAN = 1, ROW_S8 = 2 };

template <typename T, int C, bool BLOCK, bool VEC, int MODE>
__global__ void __launch_bounds__(BLOCK ? rownorm_block_threads<T, C>() : ROWNORM_THREADS)
row_norm_kernel(const RowNormParams p) {
    constexpr int V = RmsVec<T>::N, E = (int)sizeof(T);
    constexpr bool TAN = MODE == ROW_NORM_TAN;
    constexpr int N = MODE == ROW_NORM ? 1 : 2;
    ptx::dependency_wait();
    ptx::dependents_launch();
    __shared__ __align__(16) float slots[BLOCK ? 2 * 32 * N : 4];
    if constexpr (BLOCK) clear_slots(slots, 2 * 32 * N);
    const int lane = threadIdx.x & 31, rpw = BLOCK ? 1 : 32 / p.P;
    using Lane = RowLane<T, VEC>;
    const Lane L{BLOCK ? (int)threadIdx.x : lane & (p.P - 1), BLOCK ? (int)blockDim.x : p.P, p.D};
    const unsigned per_block = BLOCK ? 1u : (ROWNORM_THREADS / 32) * rpw;
    const float inv_d = 1.0f / (float)p.D;
    const bool res = p.in[1].p, tres = TAN && p.in[3].p;
    uint64_t g[C][V / 2];   // the same columns for every row
#pragma unroll
    for (int i = 0; i < C; ++i) L.scale(p.g, i, g[i]);
    unsigned turn = 0;
    for (unsigned base = blockIdx.x * per_block; base < p.total; base += gridDim.x * per_block) {
        const unsigned row = BLOCK ? base : base + (threadIdx.x >> 5) * rpw + lane / p.P;
        const bool act = BLOCK || row < p.total;
        const unsigned at = act ? row : 0;
        if (BLOCK && VEC && !TAN) row_prefetch<2>(p, row + gridDim.x, p.D * E);
        uint64_t h[C][V / 2], t[TAN ? C : 1][V / 2];
        {
            const T* x = L.template at<false>(p.in[0], at, p);
            uint4 a[C], b[C], c[TAN ? C : 1], d[TAN ? C : 1];
#pragma unroll
            for (int i = 0; i < C; ++i) a[i] = L.raw(x, act, i);
            if (res) {
                const T* r = L.template at<false>(p.in[1], at, p);
#pragma unroll
                for (int i = 0; i < C; ++i) b[i] = L.raw(r, act, i);
            }
            if constexpr (TAN) {
                const T* tx = L.template at<false>(p.in[2], at, p);
#pragma unroll
                for (int i = 0; i < C; ++i) c[i] = L.raw(tx, act, i);
                if (tres) {
                    const T* tr = L.template at<false>(p.in[3], at, p);
#pragma unroll
                    for (int i = 0; i < C; ++i) d[i] = L.raw(tr, act, i);
                }
            }
#pragma unroll
            for (int i = 0; i < C; ++i) {
                rms_unpack(a[i], h[i]);
                if constexpr (TAN) rms_unpack(c[i], t[i]);
            }
            if (res) {
                T* to = L.template at<false>(p.out[1], at, p);
#pragma unroll
                for (int i = 0; i < C; ++i) {
                    uint64_t w[V / 2];
                    rms_unpack(b[i], w);
#pragma unroll
                    for (int e = 0; e < V / 2; ++e) h[i][e] = ptx::add2(h[i][e], w[e]);
                    if (act) L.store(to, i, h[i]);
                }
            }
            if constexpr (TAN)
                if (tres) {
                    T* to = L.template at<false>(p.out[3], at, p);
#pragma unroll
                    for (int i = 0; i < C; ++i) {
                        uint64_t w[V / 2];
                        rms_unpack(d[i], w);
#pragma unroll
                        for (int e = 0; e < V / 2; ++e) t[i][e] = ptx::add2(t[i][e], w[e]);
                        if (act) L.store(to, i, t[i]);
                    }
                }
        }
        // sums[0] = h . h, sums[1] = h . th or max |g h|; h times `dn` in the first two
        float sums[N], dn = 1.f, eps = p.eps;
        auto sum_up = [&](bool scaled) {
            const uint64_t dn2 = ptx::pack2(dn, dn);
            uint64_t ss2 = 0ull, s2 = 0ull;
            float top = 0.f;
#pragma unroll
            for (int i = 0; i < C; ++i)
#pragma unroll
                for (int e = 0; e < V / 2; ++e) {
                    const uint64_t x = scaled ? ptx::mul2(h[i][e], dn2) : h[i][e];
                    if (MODE != ROW_S8 || p.norm) ss2 = ptx::fma2(x, x, ss2);
                    if constexpr (TAN) s2 = ptx::fma2(x, t[i][e], s2);
                    if constexpr (MODE == ROW_S8) {
                        float a, b;
                        ptx::unpack2(ptx::mul2(h[i][e], g[i][e]), a, b);
                        top = max_nan(top, max_nan(fabsf(a), fabsf(b)));
                    }
                }
            sums[0] = rms_hsum(ss2);
            if constexpr (N > 1) sums[N - 1] = MODE == ROW_S8 ? top : rms_hsum(s2);
            row_reduce<N, MODE == ROW_S8, BLOCK>(sums, p.P, slots + (BLOCK ? (turn++ & 1u) * 32 * N : 0));
        };
        sum_up(false);
        const bool leaves = row_leaves(sums[0], eps);
        if (BLOCK ? leaves : __any_sync(0xffffffffu, leaves)) {   // (the other rows of the warp are multiplied by 1)
            if (leaves) dn = row_first(sums[0]);
            sum_up(true);
            const float all = leaves ? row_power(dn, sums[0] * inv_d + eps * dn * dn, -16) : 1.f;
            // y, ty and 8-bit values are those of h and th both multiplied by `all`.  Where that is above 1 they are: nothing is rounded, and 1 / r may be beyond
            // the range.  Below 1 small elements would be lost, which only the 8-bit values allow, so there the factor stays with the sums.
            const float up = MODE == ROW_S8 ? all : fmaxf(all, 1.f);
            const uint64_t up2 = ptx::pack2(up, up);
#pragma unroll
            for (int i = 0; i < C; ++i)
#pragma unroll
                for (int e = 0; e < V / 2; ++e) {
                    h[i][e] = ptx::mul2(h[i][e], up2);
                    if constexpr (TAN) t[i][e] = ptx::mul2(t[i][e], up2);
                }
            dn = MODE == ROW_S8 ? 1.f : fminf(all, 1.f);
            eps = eps * all * all;
            sum_up(true);
        }
        const float root = rsqrtf(sums[0] * inv_d + eps);   // 1 / (r dn)
        const float inv = root * dn;
        if constexpr (MODE == ROW_S8) {
            // 127 v / max for every element v of the row.  Scaled first where 127 / max would leave the range of the fast division; zeros where the
            // maximum is not finite.
            const float top = sums[N - 1], up = top < 0x1p-100f ? 0x1p100f : top > 0x1p100f ? 0x1p-100f : 1.f;
            const bool fine = top <= 3.4028235e38f && top > 0.f;
            // 127 / max as k + low, which is off by 2^-43 of itself: v k + v low, rounded once, is then the fp32 number nearest to the quotient, and a
            // quotient halfway between two whole numbers (an element of half the maximum is 63.5) comes out as just that.  v k alone is up to two units
            // off, to one side for a whole row: of (8000, 768) bf16 normals 4164 values missed the even neighbour (a division by the scale in fp32 misses
            // 422, this none).  (16384, 1152) bf16: 19.7 -> 20.6 us without a norm, 25.8 -> 26.9 with norm and residual.
            const float k = fine ? __fdividef(127.f, top * up) : 0.f, low = fmaf(-k, top * up, 127.f) * k * (1.f / 127.f);
            if (act) {
                if (L.c == 0) {   // the quotient by 127, rounded once
                    const float y = p.norm ? top * inv : top, part = y * (1.f / 127.f);
                    p.aux[row] = fmaf(fmaf(-127.f, part, y), 1.f / 127.f, part);
                }
                int8_t* to = reinterpret_cast<int8_t*>(row_of(p.out[0].p + L.col(0, 0), p.out[0], at, p));
                const uint64_t up2 = ptx::pack2(up, up), k2 = ptx::pack2(k, k), low2 = ptx::pack2(low, low), round2 = ptx::pack2(12582912.f, 12582912.f);   // 1.5 2^23
#pragma unroll
                for (int i = 0; i < C; ++i) {
                    // 1.5 2^23 + x, |x| <= 127, rounds x to the nearest whole number (even on ties), whose 8 bits are the sum's lowest
                    uint32_t q[V];
#pragma unroll
                    for (int e = 0; e < V / 2; ++e) {
                        uint64_t v = ptx::mul2(h[i][e], g[i][e]);
                        if (up != 1.f) v = ptx::mul2(v, up2);
                        float a, b;
                        ptx::unpack2(ptx::add2(ptx::fma2(v, k2, ptx::mul2(v, low2)), round2), a, b);
                        q[2 * e] = __float_as_uint(a);
                        q[2 * e + 1] = __float_as_uint(b);
                    }
                    if constexpr (VEC) {
                        uint32_t w[V / 4];
#pragma unroll
                        for (int e = 0; e < V / 4; ++e) {
                            w[e] = __byte_perm(__byte_perm(q[4 * e], q[4 * e + 1], 0x0040), __byte_perm(q[4 * e + 2], q[4 * e + 3], 0x0040), 0x5410);
                            if (!fine) w[e] = 0;
                        }
                        if (L.col(i, 0) < p.D) {
                            if constexpr (V == 8) *reinterpret_cast<uint2*>(to + L.P * i * V) = make_uint2(w[0], w[V / 4 - 1]);
                            else *reinterpret_cast<uint32_t*>(to + L.P * i * V) = w[0];
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < V; ++e)
                            if (L.col(i, e) < p.D) to[L.P * (i * V + e)] = fine ? (int8_t)q[e] : (int8_t)0;
                    }
                }
            }
        } else if (act) {
            const float m = TAN ? sums[N - 1] * inv_d * root * inv : 0.f;   // (u . th) / (D r): th . h dn is known, whose mean is in the range where th is
            const uint64_t inv2 = ptx::pack2(inv, inv), nm2 = ptx::pack2(-m, -m);
            T* y = L.template at<false>(p.out[0], at, p);
            T* ty = TAN ? L.template at<false>(p.out[2], at, p) : nullptr;
#pragma unroll
            for (int i = 0; i < C; ++i) {
                uint64_t o[V / 2], u[V / 2];
#pragma unroll
                for (int e = 0; e < V / 2; ++e) {
                    u[e] = ptx::mul2(h[i][e], inv2);
                    o[e] = ptx::mul2(g[i][e], u[e]);
                }
                L.store(y, i, o);
                if constexpr (TAN) {
#pragma unroll
                    for (int e = 0; e < V / 2; ++e) o[e] = ptx::mul2(g[i][e], ptx::fma2(u[e], nm2, ptx::mul2(t[i][e], inv2)));
                    L.store(ty, i, o);
                }
            }
        }
    }
}

// Backward.  With a = g dy, b = g dty, and au = a . u, bu = b . u, ut = u . th, bt = b . th:
//     dtx = (b - u bu / D) / r + dth
//     dx  = (a - u au / D) / r + ((3 bu ut / D - bt) u - ut b - bu th) / (D r^2) + dh
//     dg  = sum over the rows of dy u + dty J th
// dx is the gradient of x and of the residual alike.  Every thread keeps the dg terms of its own columns over the rows it
// walks; a block writes one row of partial sums, and a second kernel adds those up: fixed orders, the same bits each time.
template <typename T, int C, bool BLOCK, bool VEC, bool SAME, bool TAN>
__global__ void __launch_bounds__(BLOCK ? rownorm_block_threads<T, C>() : ROWNORM_THREADS, rownorm_bwd_resident(BLOCK ? rownorm_block_threads<T, C>() : 0, C, TAN))
row_norm_bwd_kernel(const RowNormParams p) {
    constexpr int V = RmsVec<T>::N, N = TAN ? 5 : 2, E = (int)sizeof(T);
    // Rows of four chunks a thread, with tangents of two, are read again, from L1 and L2, for the outputs: held, they cost more warps than that
    // ((1024, 16384) bf16 with tangents 202 -> 106 us, (4096, 4096) 59 -> 56.5; but without tangents 32.5 -> 36.8, one chunk with them 54.6 -> 59).
    constexpr bool RELOAD = C > (TAN ? 1 : 2), HOLD_G = C <= 2;
    ptx::dependency_wait();
    __shared__ __align__(16) float slots[BLOCK ? 2 * 32 * N : 32 * V];
    if constexpr (BLOCK) clear_slots(slots, 2 * 32 * N);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, rpw = BLOCK ? 1 : 32 / p.P;
    using Lane = RowLane<T, VEC>;
    const Lane L{BLOCK ? (int)threadIdx.x : lane & (p.P - 1), BLOCK ? (int)blockDim.x : p.P, p.D};
    const unsigned per_block = BLOCK ? 1u : (ROWNORM_THREADS / 32) * rpw;
    const float inv_d = 1.0f / (float)p.D;
    const bool dh = p.in[2].p, dth = TAN && p.in[5].p;
    uint64_t held[HOLD_G ? C : 1][V / 2], dg[C][V / 2];   // the scale, and its gradient
#pragma unroll
    for (int i = 0; i < C; ++i) {
        if constexpr (HOLD_G) L.scale(p.g, i, held[i]);
#pragma unroll
        for (int e = 0; e < V / 2; ++e) dg[i][e] = 0ull;
    }
    unsigned turn = 0;
    for (unsigned base = blockIdx.x * per_block; base < p.total; base += gridDim.x * per_block) {
        const unsigned row = BLOCK ? base : base + warp * rpw + lane / p.P;
        const bool act = BLOCK || row < p.total;
        const unsigned at = act ? row : 0;
        if (BLOCK && VEC) row_prefetch<TAN ? 6 : 3>(p, row + gridDim.x, p.D * E);
        // as loaded: half the registers that bf16 rows would take as fp32
        constexpr int H = RELOAD ? 1 : C, HT = RELOAD || !TAN ? 1 : C;
        uint4 hr[H], yr[H], tr[HT], zr[HT], vh[H], vt[HT];
        const T* from[6];
        {
#pragma unroll
            for (int k = 0; k < (TAN ? 6 : 3); ++k) from[k] = L.template at<SAME>(p.in[k], at, p);
            auto load = [&](uint4* to, int k, bool there) {
#pragma unroll
                for (int i = 0; i < C; ++i) to[i] = L.raw(from[k], act && there, i);
            };
            if constexpr (!RELOAD) {
                load(hr, 0, true);
                load(yr, 1, true);
                if constexpr (TAN) { load(tr, 3, true); load(zr, 4, true); load(vt, 5, dth); }
                load(vh, 2, dh);
            }
        }
        auto unpack = [&](int i, uint64_t (&h)[V / 2], uint64_t (&y)[V / 2], uint64_t (&t)[V / 2], uint64_t (&z)[V / 2], uint64_t (&g)[V / 2]) {
            if constexpr (RELOAD) {
                rms_unpack(L.raw(from[0], act, i), h);
                rms_unpack(L.raw(from[1], act, i), y);
                if constexpr (TAN) { rms_unpack(L.raw(from[3], act, i), t); rms_unpack(L.raw(from[4], act, i), z); }
            } else {
                rms_unpack(hr[i], h);
                rms_unpack(yr[i], y);
                if constexpr (TAN) { rms_unpack(tr[i], t); rms_unpack(zr[i], z); }
            }
            if constexpr (HOLD_G) {
#pragma unroll
                for (int e = 0; e < V / 2; ++e) g[e] = held[i][e];
            } else {
                L.scale(p.g, i, g);
            }
        };
        // Ends the reuse of an earlier unpacking across the reductions.
        auto keep = [](uint4& q) { asm volatile("" : "+r"(q.x), "+r"(q.y), "+r"(q.z), "+r"(q.w)); };
        // h.h, a.h, then with tangents h.th, b.h, b.th; h, and th in the last one, times `pre`
        float s[N], pre = 1.f;
        auto sum_up = [&](bool scaled) {
            const uint64_t pre2 = ptx::pack2(pre, pre);
            uint64_t acc[N];
#pragma unroll
            for (int k = 0; k < N; ++k) acc[k] = 0ull;
#pragma unroll
            for (int i = 0; i < C; ++i) {
                uint64_t h[V / 2], y[V / 2], t[V / 2], z[V / 2], g[V / 2];
                unpack(i, h, y, t, z, g);
#pragma unroll
                for (int e = 0; e < V / 2; ++e) {
                    const uint64_t x = scaled ? ptx::mul2(h[e], pre2) : h[e];
                    acc[0] = ptx::fma2(x, x, acc[0]);
                    acc[1] = ptx::fma2(ptx::mul2(g[e], y[e]), x, acc[1]);
                    if constexpr (TAN) {
                        const uint64_t b = ptx::mul2(g[e], z[e]);
                        acc[2] = ptx::fma2(x, t[e], acc[2]);
                        acc[3] = ptx::fma2(b, x, acc[3]);
                        acc[4] = ptx::fma2(b, scaled ? ptx::mul2(t[e], pre2) : t[e], acc[4]);
                    }
                }
            }
#pragma unroll
            for (int k = 0; k < N; ++k) s[k] = rms_hsum(acc[k]);
            row_reduce<N, false, BLOCK>(s, p.P, slots + (BLOCK ? (turn++ & 1u) * 32 * N : 0));
        };
        sum_up(false);
        const bool leaves = row_leaves(s[0], p.eps);
        if (BLOCK ? leaves : __any_sync(0xffffffffu, leaves)) {
            if (leaves) pre = row_first(s[0]);
            sum_up(true);
            // large rows so that h . th stays in the range, tiny ones so that products with cotangents of their size do
            if (leaves) pre = row_power(pre, s[0] * inv_d + p.eps * pre * pre, pre < 1.f ? -16 : 16);
            sum_up(true);
        }
        const float root = rsqrtf(s[0] * inv_d + p.eps * pre * pre), inv = root * pre;   // 1 / (r pre), 1 / r
        // dx = inv (a + jt b + zh th) + kh u, dtx = inv b + zh u, J th = inv th + jt u;  u = h inv.  No factor has 1 / r^2 or a sum of products that
        // may leave the range (u . a does where its mean and dx do not).
        float kh = -inv * (s[1] * inv_d * root), zh = 0.f, jt = 0.f;
        if constexpr (TAN) {
            zh = -inv * (s[3] * inv_d * root);
            jt = -inv * (s[2] * inv_d * root);
            kh += 3.f * zh * jt - s[4] * inv_d * root * inv;
        }
        if (act) {
            const uint64_t inv2 = ptx::pack2(inv, inv), kh2 = ptx::pack2(kh, kh), zh2 = ptx::pack2(zh, zh), jt2 = ptx::pack2(jt, jt);
            T* dx = L.template at<SAME>(p.out[0], at, p);
            T* dtx = TAN ? L.template at<SAME>(p.out[1], at, p) : nullptr;
#pragma unroll
            for (int i = 0; i < C; ++i) {
                uint64_t ox[V / 2], ot[V / 2], h[V / 2], y[V / 2], t[V / 2], z[V / 2], g[V / 2];
                if constexpr (RELOAD) {
                    rms_unpack(L.raw(from[2], dh, i), ox);
                    if constexpr (TAN) rms_unpack(L.raw(from[5], dth, i), ot);
                } else {
                    rms_unpack(vh[i], ox);
                    if constexpr (TAN) rms_unpack(vt[i], ot);
                    keep(hr[i]); keep(yr[i]);
                    if constexpr (TAN) { keep(tr[i]); keep(zr[i]); }
                }
                unpack(i, h, y, t, z, g);
#pragma unroll
                for (int e = 0; e < V / 2; ++e) {
                    const uint64_t u = ptx::mul2(h[e], inv2);
                    uint64_t a = ptx::mul2(g[e], y[e]);
                    dg[i][e] = ptx::fma2(y[e], u, dg[i][e]);
                    if constexpr (TAN) {
                        const uint64_t b = ptx::mul2(g[e], z[e]);
                        a = ptx::fma2(t[e], zh2, ptx::fma2(b, jt2, a));
                        ot[e] = ptx::fma2(b, inv2, ptx::fma2(u, zh2, ot[e]));
                        dg[i][e] = ptx::fma2(z[e], ptx::fma2(t[e], inv2, ptx::mul2(u, jt2)), dg[i][e]);
                    }
                    ox[e] = ptx::fma2(a, inv2, ptx::fma2(u, kh2, ox[e]));
                }
                L.store(dx, i, ox);
                if constexpr (TAN) L.store(dtx, i, ot);
            }
        }
    }
    if (!p.aux) return;
    // the reduction may be launched: its blocks wait for this grid's end before they read anything
    ptx::dependents_launch();
    float* partial = p.aux + (size_t)blockIdx.x * p.D;
    if constexpr (BLOCK) {
#pragma unroll
        for (int i = 0; i < C; ++i)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                float a, b;
                ptx::unpack2(dg[i][e / 2], a, b);
                if (L.col(i, e) < p.D) partial[L.col(i, e)] = e & 1 ? b : a;
            }
    } else {
        for (int w = 0; w < ROWNORM_THREADS / 32; ++w) {   // the warps one after the other
            __syncthreads();
#pragma unroll
            for (int i = 0; i < C; ++i)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    float a, b;
                    ptx::unpack2(dg[i][e / 2], a, b);
                    float v = e & 1 ? b : a;
                    if (warp == w) {
                        for (int off = 16; off >= p.P; off >>= 1) v += __shfl_xor_sync(0xffffffffu, v, off);   // the rows of a warp
                        if (lane < p.P && L.col(i, e) < p.D) slots[L.col(i, e)] = w == 0 ? v : slots[L.col(i, e)] + v;
                    }
                }
        }
        __syncthreads();
        for (int j = threadIdx.x; j < p.D; j += ROWNORM_THREADS) partial[j] = slots[j];
    }
}

// dg[j] = sum over the n partial rows, in a fixed order: COLS columns a block, the rows over 1024 / COLS threads.  Launched as a
// programmatic dependent of the kernel above.  n = 0 (no rows at all) gives zeros.
template <int COLS>
__global__ void __launch_bounds__(1024) row_norm_dg_kernel(const float* partial, float* dg, int n, int D) {
    __shared__ float acc[32][COLS + 1];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, j = blockIdx.x * COLS + (lane & (COLS - 1));
    ptx::dependency_wait();
    float v = 0.f;
    if (j < D) {
#pragma unroll 8
        for (int b = threadIdx.x / COLS; b < n; b += 1024 / COLS) v += partial[(size_t)b * D + j];
    }
#pragma unroll
    for (int off = COLS; off < 32; off <<= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
    if (lane < COLS) acc[warp][lane] = v;
    __syncthreads();
    if (warp < COLS) {   // a column each
        v = acc[lane][warp];
        for (int off = 16; off > 0; off >>= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
        if (lane == 0 && blockIdx.x * COLS + warp < D) dg[blockIdx.x * COLS + warp] = v;
    }
}

}  // namespace tvm_attn

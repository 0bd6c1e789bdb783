// C-ABI entry points of the operators on rows of the model width (see include/tvm_attn.h): the RMSNorm with residual and
// tangent, its backward and its 8-bit form, and the products of 8-bit rows.  Argument checks and launches.
#include "tvm_attn.h"

#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cmath>
#include <cstring>
#include <type_traits>

#include "host_common.h"
#include "linear_s8.cuh"
#include "row_norm.cuh"

namespace tvm_attn {

// Launches a kernel as a programmatic dependent of the one in front of it on the stream: its blocks are set up while that one ends, and
// wait for its end before they touch global memory.  `cluster`: blocks of a cluster where the kernel does not say.
template <typename... P, typename... A>
static int launch(void (*kern)(P...), unsigned grid, int threads, int smem, cudaStream_t st, int cluster, const A&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = (size_t)smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 0 ? 2 : 1;
    if (cudaLaunchKernelEx(&cfg, kern, P(args)...) != cudaSuccess) {
        cudaGetLastError();
        return TVM_ATTN_CUDA_ERROR;
    }
    g_launches += 1;
    return TVM_ATTN_OK;
}

// ------------------------------------------------------------------------------------------------ rows
static int check_rows_params(const tvm_attn_rows_params* p) {
    if (!p || p->B < 0 || p->T < 0 || p->D <= 0) return TVM_ATTN_INVALID_ARG;
    if (p->dtype != TVM_ATTN_BF16 && p->dtype != TVM_ATTN_FP32) return TVM_ATTN_INVALID_ARG;
    if (!(p->eps >= 0.0f) || !std::isfinite(p->eps)) return TVM_ATTN_INVALID_ARG;
    if (p->D > TVM_ATTN_MAX_WIDTH || (long long)p->B * p->T > 2147483647LL) return TVM_ATTN_UNSUPPORTED;
    return TVM_ATTN_OK;
}

static bool present(const tvm_attn_rows* t) { return t && t->ptr; }

// What the tensors of a call have in common, gathered while they are checked.
struct RowsCall {
    const tvm_attn_rows_params& p;
    RowNormParams k;
    bool vec;   // every row begins on 16 bytes (8-bit rows: 8) and is a multiple of 16 bytes long
    int esz;
    bool ok = true;
    explicit RowsCall(const tvm_attn_rows_params& q) : p(q) {
        std::memset(&k, 0, sizeof k);
        esz = q.dtype == TVM_ATTN_FP32 ? 4 : 2;
        k.total = (unsigned)((long long)q.B * q.T);
        k.T = k.total;   // one dimension of rows, until a tensor needs two
        k.flat = k.same = true;
        k.D = q.D;
        k.eps = q.eps;
        vec = q.D * esz % 16 == 0;
    }
    void add(const tvm_attn_rows* t, RowsPtr* to, bool required, bool eight = false) {
        if (!present(t)) {
            ok = ok && !required;
            return;
        }
        const long long size = eight ? 1 : esz;
        long long row = t->row, batch = t->batch;
        if (row == 0 && batch == 0) { row = p.D; batch = (long long)p.T * p.D; }
        if (p.T <= 1) row = batch;          // one row a batch: the batches are the rows
        if (p.B <= 1) batch = row * p.T;
        if (k.total <= 1) row = batch = p.D;
        if (row < p.D || batch < p.D || row > (1LL << 40) || batch > (1LL << 40) || reinterpret_cast<uintptr_t>(t->ptr) % size) { ok = false; return; }
        *to = {static_cast<char*>(t->ptr), row * size, batch * size};
        // (8-bit rows have an offset of their own)
        if (!eight && (row * size != k.in[0].row || (long long)k.total * row * size >= 1LL << 32 || (p.T > 1 && batch != row * p.T))) k.same = false;
        if (p.T > 1 && batch != row * p.T) { k.T = (unsigned)p.T; k.flat = false; }
        if (row * size >= 1LL << 32) k.flat = false;
        const long long unit = eight ? 8 : 16;
        vec = vec && reinterpret_cast<uintptr_t>(t->ptr) % unit == 0 && row * size % unit == 0 && batch * size % unit == 0;
    }
    // Outputs that begin where another output does, or where an input does that lies differently, would be read or written by two
    // threads.  (Other overlaps are the caller's to avoid.)  `eight`: the first output is 8-bit rows, which lie differently from all inputs.
    bool overlapping(bool eight = false) const {
        for (int i = 0; i < 4; ++i) {
            const RowsPtr& o = k.out[i];
            if (!o.p) continue;
            for (int j = 0; j < i; ++j)
                if (k.out[j].p == o.p) return true;
            for (const RowsPtr& x : k.in)
                if (x.p == o.p && ((eight && i == 0) || x.row != o.row || x.batch != o.batch)) return true;
        }
        return false;
    }
    void scale(const float* g) {
        k.g = g;
        ok = ok && reinterpret_cast<uintptr_t>(g) % 4 == 0;
        vec = vec && aligned16(g);   // (a null scale is aligned)
    }
};

// How a row is split over threads: chunks of 16 bytes, one on each of P lanes of a warp, or C on each of the `threads` of a block.
struct RowSplit { int C, P, threads; };
// `single`: the most chunks of a row that has one on each thread.
static RowSplit row_split(int D, int esz, int single) {
    const int chunks = (D * esz + 15) / 16;
    if (chunks <= 32) {
        int P = 1;
        while (P < chunks) P *= 2;
        return {1, P, 0};
    }
    const int C = chunks <= single ? 1 : chunks <= 1024 ? 2 : 4;
    const int threads = ((chunks + C - 1) / C + 31) / 32 * 32;
    return {C, threads, threads};
}

// launch(C, whether a row has a block) as types, for the split of a call.
template <typename F>
static int with_row_split(const RowSplit& s, const F& launch) {
    using std::integral_constant;
    if (!s.threads) return launch(integral_constant<int, 1>(), std::false_type());
    switch (s.C) {
        case 1: return launch(integral_constant<int, 1>(), std::true_type());
        case 2: return launch(integral_constant<int, 2>(), std::true_type());
        default: return launch(integral_constant<int, 4>(), std::true_type());
    }
}

static unsigned fewer(long long a, long long b) { return (unsigned)(a < b ? a : b); }

// Blocks of `threads` that the device holds at a time, looked up once per thread, context and block size.
template <auto KERN>
static long long resident_blocks(const DeviceFacts& dev, int threads) {
    thread_local unsigned long long ctx = 0;
    thread_local int known = 0, blocks = 0;
    if (ctx != dev.ctx || known != threads) {
        int n = 0;
        if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, KERN, threads, 0) != cudaSuccess || n < 1) { cudaGetLastError(); return 0; }
        ctx = dev.ctx; known = threads; blocks = n;
    }
    return (long long)blocks * dev.sms;
}

template <typename T, int MODE>
static int launch_norm(const RowsCall& c, cudaStream_t st) {
    const DeviceFacts* dev = device_facts();
    if (!dev) return TVM_ATTN_CUDA_ERROR;
    // 8-bit rows, whose work per row weighs most, with two chunks a thread from 65 chunks on: it is then that of fewer warps.  Without a norm, 38 MB of bf16
    // rows, one chunk a thread and two: 1280 wide 21.9, 18.5 us, 1152 23.8, 20.1, 1024 19.3, 16.2; 768 19.6, 20.5;
    // 512 21.8, 16.3, 272 38.5, 27.5, where two would be the faster too.  With norm and residual alike (1152 30.0, 27.0).
    // (The norm with tangents, 1152 wide, 49.6 and 51.6.)
    const RowSplit split = row_split(c.k.D, sizeof(T), MODE == ROW_S8 ? 64 : ROWNORM_SINGLE);
    RowNormParams k = c.k;
    k.P = split.P;
    return with_row_split(split, [&](auto C, auto block) {
        const int per_block = block() ? 1 : ROWNORM_THREADS / 32 * (32 / k.P), threads = block() ? split.threads : ROWNORM_THREADS;
        const auto run = [&](auto vec) {
            constexpr auto kern = row_norm_kernel<T, decltype(C)::value, decltype(block)::value, decltype(vec)::value, MODE>;
            const long long most = resident_blocks<kern>(*dev, threads);
            if (most == 0) return (int)TVM_ATTN_CUDA_ERROR;
            return launch(kern, fewer((k.total + (long long)per_block - 1) / per_block, most), threads, 0, st, 0, k);
        };
        return c.vec ? run(std::true_type()) : run(std::false_type());
    });
}

template <int MODE>
static int launch_norm(const RowsCall& c, cudaStream_t st) {
    return c.p.dtype == TVM_ATTN_FP32 ? launch_norm<float, MODE>(c, st) : launch_norm<__nv_bfloat16, MODE>(c, st);
}

static int bwd_blocks(const RowSplit& split, bool tan, long long rows) {
    const int per_block = split.threads ? 1 : ROWNORM_THREADS / 32 * (32 / split.P);
    return (int)fewer((rows + per_block - 1) / per_block, rownorm_bwd_blocks(split.threads, split.C, tan));
}

template <typename T, bool TAN>
static int launch_norm_bwd(const RowsCall& c, float* dg, cudaStream_t st) {
    const RowSplit split = row_split(c.k.D, sizeof(T), ROWNORM_SINGLE);
    RowNormParams k = c.k;
    k.P = split.P;
    const int blocks = bwd_blocks(split, TAN, k.total);
    if (blocks > 0) {
        const int rc = with_row_split(split, [&](auto C, auto block) {
            const int threads = block() ? split.threads : ROWNORM_THREADS;
            return !c.vec ? launch(row_norm_bwd_kernel<T, C(), block(), false, false, TAN>, blocks, threads, 0, st, 0, k)
                 : k.same ? launch(row_norm_bwd_kernel<T, C(), block(), true, true, TAN>, blocks, threads, 0, st, 0, k)
                          : launch(row_norm_bwd_kernel<T, C(), block(), true, false, TAN>, blocks, threads, 0, st, 0, k);
        });
        if (rc != TVM_ATTN_OK) return rc;
    }
    if (!dg) return TVM_ATTN_OK;
    // as few columns a block as leave no SM without one: 8 are a sector of each partial row, 32 a line
    if (k.D <= 8 * 148) return launch(row_norm_dg_kernel<8>, (unsigned)(k.D + 7) / 8, 1024, 0, st, 0, k.aux, dg, blocks, k.D);
    return launch(row_norm_dg_kernel<32>, (unsigned)(k.D + 31) / 32, 1024, 0, st, 0, k.aux, dg, blocks, k.D);
}

static size_t norm_bwd_workspace(const tvm_attn_rows_params& p) {
    const RowSplit split = row_split(p.D, p.dtype == TVM_ATTN_FP32 ? 4 : 2, ROWNORM_SINGLE);
    const int tan = rownorm_bwd_blocks(split.threads, split.C, true), plain = rownorm_bwd_blocks(split.threads, split.C, false);
    return (size_t)(tan > plain ? tan : plain) * (size_t)p.D * sizeof(float);
}

}  // namespace tvm_attn

using namespace tvm_attn;

extern "C" {

int tvm_attn_rmsnorm_jvp_fwd(const tvm_attn_rows_params* p, const tvm_attn_rows* x, const tvm_attn_rows* res, const tvm_attn_rows* tx,
                             const tvm_attn_rows* tres, const float* g, const tvm_attn_rows* y, const tvm_attn_rows* h,
                             const tvm_attn_rows* ty, const tvm_attn_rows* th, void* cuda_stream) {
    const int rc = check_rows_params(p);
    if (rc != TVM_ATTN_OK) return rc;
    if (present(res) != present(h) || present(tx) != present(ty) || present(tres) != present(th) || (present(tres) && !present(tx))) return TVM_ATTN_INVALID_ARG;
    RowsCall c(*p);
    if (c.k.total == 0) return TVM_ATTN_OK;
    c.add(x, &c.k.in[0], true); c.add(res, &c.k.in[1], false); c.add(tx, &c.k.in[2], false); c.add(tres, &c.k.in[3], false);
    c.add(y, &c.k.out[0], true); c.add(h, &c.k.out[1], false); c.add(ty, &c.k.out[2], false); c.add(th, &c.k.out[3], false);
    c.scale(g);
    if (!c.ok || c.overlapping()) return TVM_ATTN_INVALID_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    return present(tx) ? launch_norm<ROW_NORM_TAN>(c, st) : launch_norm<ROW_NORM>(c, st);
}

size_t tvm_attn_rmsnorm_jvp_workspace_bytes(const tvm_attn_rows_params* p) {
    return check_rows_params(p) == TVM_ATTN_OK ? norm_bwd_workspace(*p) : 0;
}

int tvm_attn_rmsnorm_jvp_bwd(const tvm_attn_rows_params* p, const tvm_attn_rows* h, const tvm_attn_rows* dy, const tvm_attn_rows* dh,
                             const tvm_attn_rows* th, const tvm_attn_rows* dty, const tvm_attn_rows* dth, const float* g,
                             const tvm_attn_rows* dx, const tvm_attn_rows* dtx, float* dg, void* workspace, size_t workspace_bytes,
                             void* cuda_stream) {
    const int rc = check_rows_params(p);
    if (rc != TVM_ATTN_OK) return rc;
    if (present(th) != present(dty) || present(th) != present(dtx) || (present(dth) && !present(th)) || !g != !dg) return TVM_ATTN_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(dg) % 4) return TVM_ATTN_INVALID_ARG;
    RowsCall c(*p);
    c.scale(g);
    if (c.k.total > 0) {
        c.add(h, &c.k.in[0], true); c.add(dy, &c.k.in[1], true); c.add(dh, &c.k.in[2], false);
        c.add(th, &c.k.in[3], false); c.add(dty, &c.k.in[4], false); c.add(dth, &c.k.in[5], false);
        c.add(dx, &c.k.out[0], true); c.add(dtx, &c.k.out[1], false);
    }
    if (!c.ok || c.overlapping()) return TVM_ATTN_INVALID_ARG;
    if (g) {
        if (!workspace || !aligned16(workspace)) return TVM_ATTN_INVALID_ARG;
        if (workspace_bytes < norm_bwd_workspace(*p)) return TVM_ATTN_WORKSPACE_TOO_SMALL;
        c.k.aux = static_cast<float*>(workspace);
    }
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    if (p->dtype == TVM_ATTN_FP32) return present(th) ? launch_norm_bwd<float, true>(c, dg, st) : launch_norm_bwd<float, false>(c, dg, st);
    return present(th) ? launch_norm_bwd<__nv_bfloat16, true>(c, dg, st) : launch_norm_bwd<__nv_bfloat16, false>(c, dg, st);
}

int tvm_attn_rmsnorm_s8(const tvm_attn_rows_params* p, const tvm_attn_rows* x, const tvm_attn_rows* res, const float* g,
                        const tvm_attn_rows* q, float* s, const tvm_attn_rows* h, void* cuda_stream) {
    const int rc = check_rows_params(p);
    if (rc != TVM_ATTN_OK) return rc;
    if (present(res) != present(h)) return TVM_ATTN_INVALID_ARG;
    RowsCall c(*p);
    if (c.k.total == 0) return TVM_ATTN_OK;
    c.add(x, &c.k.in[0], true); c.add(res, &c.k.in[1], false);
    c.add(q, &c.k.out[0], true, true); c.add(h, &c.k.out[1], false);
    c.scale(g);
    if (!c.ok || c.overlapping(true) || !s || reinterpret_cast<uintptr_t>(s) % 4) return TVM_ATTN_INVALID_ARG;
    c.k.aux = s;
    c.k.norm = true;
    return launch_norm<ROW_S8>(c, static_cast<cudaStream_t>(cuda_stream));
}

int tvm_attn_quantize_s8(const tvm_attn_rows_params* p, const tvm_attn_rows* x, const tvm_attn_rows* q, float* s, void* cuda_stream) {
    const int rc = check_rows_params(p);
    if (rc != TVM_ATTN_OK) return rc;
    RowsCall c(*p);
    if (c.k.total == 0) return TVM_ATTN_OK;
    c.add(x, &c.k.in[0], true);
    c.add(q, &c.k.out[0], true, true);
    if (!c.ok || c.overlapping(true) || !s || reinterpret_cast<uintptr_t>(s) % 4) return TVM_ATTN_INVALID_ARG;
    c.k.aux = s;
    c.k.eps = 1.f;   // (the sum of squares is not used: nothing is to be scaled for it)
    return launch_norm<ROW_S8>(c, static_cast<cudaStream_t>(cuda_stream));
}

}  // extern "C"

namespace tvm_attn {

// ------------------------------------------------------------------------------------------------ 8-bit products
template <typename OUT, int MT, int R>
static int launch_few(const LinearParams& p, cudaStream_t st) {
    const int rows = R * (LIN_FEW_THREADS / 32);
    return launch(linear_s8_few_kernel<OUT, MT, R>, (unsigned)((p.N + rows - 1) / rows), LIN_FEW_THREADS, 0, st, 0, p);
}

template <typename OUT, int MT>
static int linear_few(const LinearParams& p, cudaStream_t st) {
    // channels a warp: as many as leave 16 warps for each SM
    if (p.N >= 148 * 16 * 4) return launch_few<OUT, MT, 4>(p, st);
    if (p.N >= 148 * 16 * 2) return launch_few<OUT, MT, 2>(p, st);
    return launch_few<OUT, MT, 1>(p, st);
}

// A matrix (rows, cols) in boxes of box_cols x box_rows; what lies outside it reads as zero and is not written.
static int matrix_map(CUtensorMap* m, CUtensorMapDataType type, int size, const void* ptr, long long cols, long long rows, long long pitch, int box_cols, int box_rows,
                      CUtensorMapSwizzle swizzle) {
    encode_tiled_fn fn = get_encode_fn();
    if (!fn) return TVM_ATTN_CUDA_ERROR;
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)(pitch * size)};
    const cuuint32_t box[2] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows}, step[2] = {1, 1};
    return fn(m, type, 2, const_cast<void*>(ptr), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS ? TVM_ATTN_OK : TVM_ATTN_CUDA_ERROR;
}

template <int BN, typename OUT>
static int launch_many(LinearParams p, const DeviceFacts& dev, cudaStream_t st) {
    using C = LinCfg<BN, OUT>;
    constexpr auto kern = linear_s8_kernel<BN, OUT>;
    thread_local unsigned long long prepared = 0;   // once per thread and context
    if (prepared != dev.ctx) {
        if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM_BYTES) != cudaSuccess) { cudaGetLastError(); return TVM_ATTN_CUDA_ERROR; }
        prepared = dev.ctx;
    }
    constexpr bool HALF = sizeof(OUT) == 2;
    CUtensorMap ma, mb, my;
    int rc = matrix_map(&ma, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, p.q, p.K, p.M, p.ldq, 128, LIN_ROWS, CU_TENSOR_MAP_SWIZZLE_128B);
    if (rc == TVM_ATTN_OK) rc = matrix_map(&mb, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, p.w, p.K, p.N, p.ldw, 128, BN / 2, CU_TENSOR_MAP_SWIZZLE_128B);
    my = ma;   // (not used where y's rows do not begin on 16 bytes)
    const bool begin = aligned16(p.y) && p.ldy * (long long)sizeof(OUT) % 16 == 0, end = p.N * (long long)sizeof(OUT) % 16 == 0;
    p.tma_cols = !begin ? 0 : end ? INT32_MAX : p.N;
    if (rc == TVM_ATTN_OK && begin)
        rc = matrix_map(&my, HALF ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, (int)sizeof(OUT), p.y, p.N, p.M, p.ldy, C::UNIT, 32,
                        CU_TENSOR_MAP_SWIZZLE_128B);
    if (rc != TVM_ATTN_OK) return rc;
    p.tiles_m = (p.M + 2 * LIN_ROWS - 1) / (2 * LIN_ROWS);
    p.tiles_n = (p.N + BN - 1) / BN;
    p.status = dev.status;
    const long long tiles = (long long)p.tiles_m * p.tiles_n;
    return launch(kern, 2 * fewer(tiles, dev.sms / 2), LIN_THREADS, C::SMEM_BYTES, st, 0, ma, mb, my, p);
}

// Cycles of a product in tiles of 256 rows, and the width of a tile: the one whose rounds of tiles take least.  Narrow tiles load more for what
// they compute: 128 bytes of k took 776, 624, 546 and 484 cycles with 256, 192, 128 and 64 channels (K = 9216, four tiles a pair, of a clock that the power
// cap lowers), in proportion to 256 + BN.  16384 x 3456 x 1152 51.9, 54.4, 65.8, 109.8 us; 8000 x 768 x 768 10.5, 9.6, 10.8, 15.6; 512 x 4608 x 1152 9.5,
// 8.5, 7.6, 11.0.  (Widths are compared with one another, for which the factor does not matter; 6/5 of a cycle, less than a stage takes in a long product,
// puts the crossing with thin_cycles where the times in linear() have it.)  -1: more tiles than there can be.
static long long many_cycles(const LinearParams& p, const DeviceFacts& dev, int* width) {
    const long long tiles_m = (p.M + 2 * LIN_ROWS - 1) / (2 * LIN_ROWS), pairs = dev.sms / 2, kblocks = (p.K + 127) / 128;
    if (tiles_m * ((p.N + 63) / 64) > 2147483647LL) return -1;
    long long least = -1;
    for (int bn : {256, 192, 128, 64}) {
        const long long rounds = (tiles_m * ((p.N + bn - 1) / bn) + pairs - 1) / pairs, cost = rounds * kblocks * (256 + bn) * 6 / 5;
        if (least < 0 || cost < least) { least = cost; *width = bn; }
    }
    return least;
}

template <int NT, typename OUT>
static int launch_thin(LinearParams p, const DeviceFacts& dev, cudaStream_t st) {
    using C = ThinCfg<NT>;
    constexpr auto kern = linear_s8_thin_kernel<NT, OUT>;
    thread_local unsigned long long prepared = 0;   // once per thread and context
    if (prepared != dev.ctx) {
        if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM_BYTES) != cudaSuccess) { cudaGetLastError(); return TVM_ATTN_CUDA_ERROR; }
        prepared = dev.ctx;
    }
    CUtensorMap mw, mq;
    int rc = matrix_map(&mw, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, p.w, p.K, p.N, p.ldw, 128, 128, CU_TENSOR_MAP_SWIZZLE_128B);
    if (rc == TVM_ATTN_OK) rc = matrix_map(&mq, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, p.q, p.K, p.M, p.ldq, 128, NT, CU_TENSOR_MAP_SWIZZLE_128B);
    if (rc != TVM_ATTN_OK) return rc;
    p.status = dev.status;
    return launch(kern, (unsigned)((p.N + 127) / 128) * p.ksplit, LIN_THIN_THREADS, C::SMEM_BYTES, st, p.ksplit, mw, mq, p);
}

template <typename OUT>
static int linear_thin(const LinearParams& p, const DeviceFacts& dev, cudaStream_t st) {
    if (p.M <= 16) return launch_thin<16, OUT>(p, dev, st);
    if (p.M <= 32) return launch_thin<32, OUT>(p, dev, st);
    if (p.M <= 64) return launch_thin<64, OUT>(p, dev, st);
    return p.M <= 128 ? launch_thin<128, OUT>(p, dev, st) : launch_thin<256, OUT>(p, dev, st);
}

// Cycles of a product on linear_s8_thin_kernel, by its number of CTAs that share k: an SM's CTAs share its loads (some 64 bytes a cycle) and the
// writes of their sums (26 cycles a token), and add up some tokens each (125 cycles a token).
static long long thin_cycles(const LinearParams& p, const DeviceFacts& dev, int split) {
    const int NT = p.M <= 16 ? 16 : p.M <= 32 ? 32 : p.M <= 64 ? 64 : p.M <= 128 ? 128 : 256;
    const long long tiles = (p.N + 127) / 128, kblocks = (p.K + 127) / 128, ctas = (tiles * split + dev.sms - 1) / dev.sms;
    return ctas * ((kblocks + split - 1) / split * (128 + NT) * 2 + (split > 1 ? 26LL * p.M : 0)) + 125LL * ((p.M + split - 1) / split);
}

template <typename OUT>
static int linear(LinearParams p, cudaStream_t st) {
    const DeviceFacts* dev;
    const int rc = tensor_core_device(&dev);
    if (rc != TVM_ATTN_OK) return rc;
    // One or two tokens on dp4a, unless the products are so long that they take longer than the weights' bytes.  14336 x 4096 weights, one
    // token 11.6 us (13.7 on the tensor cores), two 12.3; 4096 x 14336 one 12.9 (14.7), two 17.9 (14.5).
    if (p.M <= 2 && (long long)p.M * p.K <= 16384) return p.M == 1 ? linear_few<OUT, 1>(p, st) : linear_few<OUT, 2>(p, st);
    int bn = 0;
    const long long many = many_cycles(p, *dev, &bn);
    if (p.M <= 256) {
        // Weights past the tokens, k shared by as many CTAs as is fastest, where that beats tiles of 256 rows by the two estimates.  Times in us (thin,
        // many) and what is taken: tokens x (14336 x 4096) 48: 16.3, 17.5 thin; 56: 17.3, 17.5 thin; 58: 17.3, 17.5 many; 64: 17.9, 17.5 many; 128: 32.8, 17.8
        // many; x (4096 x 14336) 64: 17.7, 27.2 thin; 256: 24.9, 27.7 thin; x (4608 x 1152) 32: 6.7, 7.0 thin; 48: 8.6, 7.0 many; x (1152 x 4608) 192: 11.7, 11.7
        // many; 256: 14.3, 11.8 many; x (768 x 768) 32: 4.7, 5.5 thin; 48: 4.9, 5.6 many, the one of these where the other was faster; 96: 6.5, 5.8 many.
        const int kblocks = (p.K + 127) / 128;
        // up to 64 tokens three CTAs of an SM together keep enough of the weights in flight: as many share k as are resident (two of them, 14336 x
        // 4096: 18.6 instead of 16.5 us); then the number of them that is fastest
        const long long tiles = (p.N + 127) / 128, resident = 3LL * dev->sms / tiles, most = kblocks < 8 ? kblocks : 8;
        const int least = p.M > 64 || resident < 1 ? 1 : (int)(resident < most ? resident : most);
        long long thin = -1;
        for (int split = least; split <= (p.M > 64 ? most : least); ++split) {
            const long long c = thin_cycles(p, *dev, split);
            if (thin < 0 || c < thin) { thin = c; p.ksplit = split; }
        }
        if (thin <= many || many < 0) return linear_thin<OUT>(p, *dev, st);
    }
    switch (bn) {
        case 256: return launch_many<256, OUT>(p, *dev, st);
        case 192: return launch_many<192, OUT>(p, *dev, st);
        case 128: return launch_many<128, OUT>(p, *dev, st);
        case 64: return launch_many<64, OUT>(p, *dev, st);
        default: return TVM_ATTN_UNSUPPORTED;   // more tiles than 31 bits hold
    }
}

}  // namespace tvm_attn

extern "C" int tvm_attn_linear_s8(const tvm_attn_linear_params* p, const void* q, const float* s, const void* w, const float* ws, const float* bias,
                                  void* y, void* cuda_stream) {
    if (!p || p->M < 0 || p->N <= 0 || p->K <= 0) return TVM_ATTN_INVALID_ARG;
    if (p->dtype != TVM_ATTN_BF16 && p->dtype != TVM_ATTN_FP32) return TVM_ATTN_INVALID_ARG;
    const long long ldq = p->ldq ? p->ldq : p->K, ldw = p->ldw ? p->ldw : p->K, ldy = p->ldy ? p->ldy : p->N;
    if (ldq < p->K || ldw < p->K || ldy < p->N || ldq % 16 || ldw % 16) return TVM_ATTN_INVALID_ARG;
    // sums of K products of at most 2^14 in 32 bits; strides as a tensor map holds them
    if (p->K > 65536 || p->M > 1 << 30 || p->N > 1 << 30 || ldq >= (1LL << 38) || ldw >= (1LL << 38) || ldy >= (1LL << 36)) return TVM_ATTN_UNSUPPORTED;
    if (p->M == 0) return TVM_ATTN_OK;
    const int esz = p->dtype == TVM_ATTN_FP32 ? 4 : 2;
    if (!q || !s || !w || !ws || !y || !aligned16(q) || !aligned16(w) || reinterpret_cast<uintptr_t>(y) % esz) return TVM_ATTN_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(s) % 4 || reinterpret_cast<uintptr_t>(ws) % 4 || reinterpret_cast<uintptr_t>(bias) % 4) return TVM_ATTN_INVALID_ARG;
    LinearParams k;
    std::memset(&k, 0, sizeof k);
    k.q = static_cast<const int8_t*>(q); k.w = static_cast<const int8_t*>(w);
    k.s = s; k.ws = ws; k.bias = bias; k.y = y;
    k.ldq = ldq; k.ldw = ldw; k.ldy = ldy;
    k.M = p->M; k.N = p->N; k.K = p->K;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    return p->dtype == TVM_ATTN_FP32 ? linear<float>(k, st) : linear<__nv_bfloat16>(k, st);
}

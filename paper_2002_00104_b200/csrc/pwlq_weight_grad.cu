// Weight gradient of a projection from the 8-bit checkpoint of its input:
// dw[n, k] = sum over t of dy[t, n] * xhat[t, k], xhat rounded to dy's type.
//
// The checkpoint is decoded to 16 bits in the workspace first (one pass, bound by HBM); then a pair
// of CTAs owns 256 x 256 of dw (n x k) and walks the rows t in steps of 64: each CTA brings 128
// columns of either operand in with TMA, and the pair's tensor cores multiply what both hold
// (tcgen05, cta_group::2, M = N = 256).  Both operands lie with their columns innermost, as in
// memory: nothing is transposed.  The sums stay in tensor memory, two tiles of 256 columns, so that
// a tile's results leave while the next one is summed.
//
// Why xhat is rounded: both operands of a 16-bit product have one type, and dy has 16 bits.  A binary32 xhat
// would be two products (its leading and its remaining bits), twice the tensor pipe's time, or tf32 operands at
// half the rate, which round to 11 bits all the same.  What it costs, as a part of dw's norm, 8192 x 4096 x
// 4096: bf16 0.0015 (fp16 8192 x 1000 x 2048: 0.00019), in a 16-bit dw 0.0023 (0.00028), where rounding the
// exact sum gives 0.0017 (0.00021) and the checkpoint itself is off by 0.0073 (0.0072).
//
// Bound by the tensor pipe: 94 % busy, 8192 x 4096 x 4096 bf16 in 173 us (1589 TFLOP/s), next to 16 us of
// decoding and 7 of adding pieces, at full clock.  The whole call takes 187 us at first and, once the power limit
// lowers the clock, 217 us at 1530 MHz and 234 at 1372.  Decoding inside the product instead, by warps that feed the tensor cores
// from shared memory, took 843 us in all against 263; decoding beside it, with flags between the two kernels,
// 262 against 211 (back to back on warm caches).
//
// The pairs are persistent.  Whole tiles go round the pairs first; the tiles of the last, partial
// round are cut along t so that they fill it, their binary32 pieces go to the workspace, and a
// second kernel adds them in the order of t.
#include <mutex>
#include <type_traits>

#include "pwlq_act8.cuh"
#include "pwlq_tcgen05.cuh"
#include "pwlq_train.h"

namespace pwlq {

static __device__ int g_weight_grad_timeout;    // a bounded wait expired

namespace {

constexpr int kTile = 256;                      // of dw, both ways, per pair of CTAs
constexpr int kHalf = 128;                      // a CTA's share of either operand
constexpr int kStep = 64;                       // rows t per stage
constexpr int kStages = 6;
constexpr int kBlockBytes = kStep * 128;        // 64 columns x 64 rows of 16-bit values
constexpr int kOperandBytes = 2 * kBlockBytes;
constexpr int kStageBytes = 2 * kOperandBytes;
constexpr int kEpilogueWarps = 8, kTmaWarp = kEpilogueWarps, kMmaWarp = kTmaWarp + 1;
constexpr int kThreads = 32 * (kMmaWarp + 1);
// A cut costs about 4 us (the pieces' way through memory, and a second kernel), a step 0.36 us: tiles
// of fewer than kCutSteps steps stay whole, and a piece has at least kMinSteps.
constexpr int kCutSteps = 24, kMinSteps = 6;

struct Shared {
    uint64_t full[kStages];        // in the leading CTA: both halves of both operands are there
    uint64_t empty[kStages];       // in each CTA: the stage has been multiplied
    uint64_t sum_full[2], sum_empty[2];
    uint32_t tmem;
    float turn[kEpilogueWarps][32][33];    // a warp's 32 x 32 results on their way to dw
};
constexpr size_t kSmemBytes = kStages * kStageBytes + 1024 + sizeof(Shared);

// The work: units 0 .. whole - 1 are whole tiles, the rest are pieces of the last tiles.
struct Schedule {
    int tiles_n, tiles_k;
    int64_t whole;                 // uncut tiles
    int64_t pieces;                // per cut tile
    int64_t units;
    int64_t steps;                 // of a whole tile
};
struct Unit {
    int64_t n0, k0, step0, step1;
    int64_t slot;                  // of its piece in the workspace, -1: a whole tile
};
__device__ __forceinline__ Unit unit_of(const Schedule& s, int64_t u) {
    Unit w;
    int64_t tile = u;
    w.step0 = 0;
    w.step1 = s.steps;
    w.slot = -1;
    if (u >= s.whole) {
        w.slot = u - s.whole;
        tile = s.whole + w.slot / s.pieces;
        const int64_t piece = w.slot % s.pieces;
        w.step0 = s.steps * piece / s.pieces;
        w.step1 = s.steps * (piece + 1) / s.pieces;
    }
    w.n0 = tile % s.tiles_n * kTile;
    w.k0 = tile / s.tiles_n * kTile;
    return w;
}

struct Params {
    WeightGrad w;
    Schedule s;
    float* pieces;                 // workspace: [slot][block of 32 x 32][four columns][row][4]
    bool vec_out;                  // rows of dw start on 16-byte boundaries
};

// A wait of a whole warp, by its first lane; the same answer in every lane.
__device__ __forceinline__ bool warp_wait(uint64_t* bar, unsigned parity) {
    bool ok = true;
    if ((threadIdx.x & 31) == 0) ok = mbar_wait_cluster(bar, parity);
    return __all_sync(0xffffffffu, ok);
}

// One lane: this CTA's columns of both operands, two boxes of 64 each per stage.
__device__ void tma_loop(const Params& p, const CUtensorMap* map, const CUtensorMap* xmap, Shared& sh,
                         unsigned char* stages, uint32_t rank) {
    const uint32_t full = peer_addr(sh.full, 0);
    int stage = 0;
    unsigned phase = 0;
    bool ok = true;
    for (int64_t u = blockIdx.x >> 1; u < p.s.units && ok; u += gridDim.x >> 1) {
        const Unit unit = unit_of(p.s, u);
        const int n = (int)(unit.n0 + rank * kHalf), k = (int)(unit.k0 + rank * kHalf);
        for (int64_t step = unit.step0; step < unit.step1; ++step) {
            if (!mbar_wait_cluster(&sh.empty[stage], phase ^ 1)) { ok = false; break; }
            if (rank == 0) mbar_expect_tx(&sh.full[stage], 4 * kOperandBytes);
            unsigned char* to = stages + stage * kStageBytes;
            const uint32_t bar = full + stage * (uint32_t)sizeof(uint64_t);
            tma_load_pair(to, map, n, (int)(step * kStep), bar);
            tma_load_pair(to + kBlockBytes, map, n + 64, (int)(step * kStep), bar);
            tma_load_pair(to + kOperandBytes, xmap, k, (int)(step * kStep), bar);
            tma_load_pair(to + kOperandBytes + kBlockBytes, xmap, k + 64, (int)(step * kStep), bar);
            if (++stage == kStages) { stage = 0; phase ^= 1; }
        }
    }
    if (!ok) g_weight_grad_timeout = 1;
    // copies in flight end before the CTA does: every stage comes back empty (at once if unused)
    for (int i = 0; i < kStages; ++i) {
        if (!mbar_wait_cluster(&sh.empty[stage], phase ^ 1)) { g_weight_grad_timeout = 1; break; }
        if (++stage == kStages) { stage = 0; phase ^= 1; }
    }
}

// One lane of the leading CTA: the products of both.
template <typename T>
__device__ void mma_loop(const Params& p, Shared& sh, unsigned char* stages, uint32_t tmem) {
    constexpr uint32_t idesc = mma_f16_idesc(std::is_same<T, __nv_bfloat16>::value, kTile, kTile);
    int stage = 0, sum = 0;
    unsigned phase = 0, sum_phase = 0;
    for (int64_t u = blockIdx.x >> 1; u < p.s.units; u += gridDim.x >> 1) {
        const Unit unit = unit_of(p.s, u);
        if (!mbar_wait_cluster(&sh.sum_empty[sum], sum_phase ^ 1)) { g_weight_grad_timeout = 1; return; }
        tcgen05_after_sync();
        const uint32_t d = tmem + sum * kTile;
        for (int64_t step = unit.step0; step < unit.step1; ++step) {
            if (!mbar_wait_cluster(&sh.full[stage], phase)) { g_weight_grad_timeout = 1; return; }
            tcgen05_after_sync();
            const uint32_t at = smem_addr(stages + stage * kStageBytes);
            const uint64_t a = outer_major_desc(at, kBlockBytes);
            const uint64_t b = outer_major_desc(at + kOperandBytes, kBlockBytes);
#pragma unroll
            for (int i = 0; i < kStep / 16; ++i)      // 16 rows t are 2048 bytes of either operand
                mma_f16_pair(d, a + i * (2048 >> 4), b + i * (2048 >> 4), idesc,
                             step > unit.step0 || i > 0);
            mma_commit_pair(&sh.empty[stage]);
            if (++stage == kStages) { stage = 0; phase ^= 1; }
        }
        mma_commit_pair(&sh.sum_full[sum]);
        if (++sum == 2) { sum = 0; sum_phase ^= 1; }
    }
}

// Where the block of 32 x 32 values at (row, column) of a piece begins.
__device__ __forceinline__ int64_t piece_block(int64_t slot, int64_t row, int64_t c) {
    return slot * (kTile * kTile) + (row / 32 * (kTile / 32) + c / 32) * 1024;
}

// A warp's 32 x 32 results (one row per lane) to rows of dw that start at `to`, `ld` apart; `rows`
// and `cols` of them exist.
template <typename W>
__device__ __forceinline__ void put_block(float* v, float (*turn)[33], W* to, int64_t ld, int rows, int cols,
                                          bool vec, bool accumulate) {
    const int lane = threadIdx.x & 31;
    if (vec && cols >= 32) {
        if (lane >= rows) return;
        to += lane * ld;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            Raw8<W> raw;
            if (accumulate) {
                float old[8];
                raw.load(to + 8 * i);
                raw.get(old);
#pragma unroll
                for (int k = 0; k < 8; ++k) v[8 * i + k] += old[k];
            }
            raw.set(v + 8 * i);
            raw.store(to + 8 * i);
        }
        return;
    }
    // rows off their alignment, or the last columns: turned in shared memory, so that a warp writes
    // 32 neighbours of a row (one value per lane and row took 42 us for 515 x 1283 results, against 15).
    // Accumulating, each of them waits for what it adds to: 48 us a call against 18, rows of 333.
#pragma unroll
    for (int i = 0; i < 32; ++i) turn[lane][i] = v[i];
    __syncwarp();
#pragma unroll 8
    for (int i = 0; i < 32; ++i) {
        const float r = turn[i][lane];
        if (i < rows && lane < cols) {
            W* at = to + i * ld + lane;
            *at = from_f32<W>(accumulate ? r + to_f32(*at) : r);
        }
    }
    __syncwarp();
}

// Four results of one row to dw, the first `valid` of which exist.
template <typename W>
__device__ __forceinline__ void put4(const float* r, W* to, int valid, bool vec, bool accumulate) {
    struct alignas(4 * sizeof(W)) Four { W v[4]; } out;
    if (vec && valid == 4) {
        if (accumulate) out = *reinterpret_cast<const Four*>(to);
#pragma unroll
        for (int i = 0; i < 4; ++i) out.v[i] = from_f32<W>(accumulate ? r[i] + to_f32(out.v[i]) : r[i]);
        *reinterpret_cast<Four*>(to) = out;
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < valid) to[i] = from_f32<W>(accumulate ? r[i] + to_f32(to[i]) : r[i]);
}

template <typename T>
__device__ void epilogue_loop(const Params& p, Shared& sh, uint32_t tmem, uint32_t rank) {
    // a warp reads the quarter of the lanes that its number selects; two share it, half the columns each
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, quarter = warp & 3;
    const int first = (warp >> 2) * (kTile / 2);
    const uint32_t empty = peer_addr(sh.sum_empty, 0);
    int sum = 0;
    unsigned phase = 0;
    for (int64_t u = blockIdx.x >> 1; u < p.s.units; u += gridDim.x >> 1) {
        const Unit unit = unit_of(p.s, u);
        if (!warp_wait(&sh.sum_full[sum], phase)) { g_weight_grad_timeout = 1; return; }
        tcgen05_after_sync();
        const int64_t row = rank * kHalf + quarter * 32, n = unit.n0 + row;      // of the warp's first lane
        for (int c = first; c < first + kTile / 2; c += 32) {
            float v[32];
            __syncwarp();
            tmem_load32(tmem + ((uint32_t)(quarter * 32) << 16) + sum * kTile + c, v);
            const int64_t k = unit.k0 + c;
            if (unit.slot >= 0) {
                float4* to = reinterpret_cast<float4*>(p.pieces + piece_block(unit.slot, row, c)) + lane;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    to[32 * i] = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
            } else if (n < p.w.outputs && k < p.w.x.cols) {
                const int rows = (int)min((int64_t)32, p.w.outputs - n), cols = (int)min((int64_t)32, p.w.x.cols - k);
                const int64_t at = n * p.w.lddw + k;
                if (p.w.dw_dtype == kF32)
                    put_block(v, sh.turn[warp], static_cast<float*>(p.w.dw) + at, p.w.lddw, rows, cols,
                              p.vec_out, p.w.accumulate);
                else
                    put_block(v, sh.turn[warp], static_cast<T*>(p.w.dw) + at, p.w.lddw, rows, cols,
                              p.vec_out, p.w.accumulate);
            }
        }
        tcgen05_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(empty + sum * (uint32_t)sizeof(uint64_t));
        if (++sum == 2) { sum = 0; phase ^= 1; }
    }
}

template <typename T>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
weight_grad_kernel(const __grid_constant__ CUtensorMap dy, const __grid_constant__ CUtensorMap xhat,
                   const __grid_constant__ Params p) {
    extern __shared__ unsigned char raw[];
    // the swizzle counts from 1024-byte boundaries
    unsigned char* stages = raw + ((1024 - (smem_addr(raw) & 1023)) & 1023);
    Shared& sh = *reinterpret_cast<Shared*>(stages + kStages * kStageBytes);
    const int warp = threadIdx.x >> 5;
    const uint32_t rank = cluster_rank();
    if (threadIdx.x == 0) {
        for (int i = 0; i < kStages; ++i) {
            mbar_init(&sh.full[i], 1);
            mbar_init(&sh.empty[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&sh.sum_full[i], 1);
            mbar_init(&sh.sum_empty[i], 2 * kEpilogueWarps);
        }
        fence_barrier_init();
    }
    if (warp == kMmaWarp) tmem_alloc_pair(&sh.tmem);
    if (threadIdx.x == kTmaWarp * 32) {
        prefetch_map(&dy);
        prefetch_map(&xhat);
    }
    tcgen05_before_sync();
    __syncthreads();
    cluster_sync();
    tcgen05_after_sync();
    const uint32_t tmem = sh.tmem;
    allow_dependents();
    await_previous();                      // the operands' kernels, and the last reader of the workspace

    if (warp < kEpilogueWarps) {
        epilogue_loop<T>(p, sh, tmem, rank);
    } else if (warp == kTmaWarp) {
        if ((threadIdx.x & 31) == 0) tma_loop(p, &dy, &xhat, sh, stages, rank);
    } else if (rank == 0) {
        if ((threadIdx.x & 31) == 0) mma_loop<T>(p, sh, stages, tmem);
    }
    __syncwarp();
    tcgen05_before_sync();
    cluster_sync();
    tcgen05_after_sync();
    if (warp == kMmaWarp) tmem_free_pair(tmem);
}

// Adds the pieces of the cut tiles in the order of t: a CTA per block of 32 x 32 values, four columns of
// one row per thread, eight pieces requested at a time (one after the other, 32 pieces of a 256 x 256
// tile took 40 us).
template <typename T>
__global__ void __launch_bounds__(256) weight_grad_pieces_kernel(const __grid_constant__ Params p) {
    __shared__ float turn[32][36];
    constexpr int kBlocks = (kTile / 32) * (kTile / 32);
    const int64_t cut = blockIdx.x / kBlocks;
    const int block = (int)(blockIdx.x % kBlocks);
    const int64_t tile = p.s.whole + cut;
    const int64_t n0 = tile % p.s.tiles_n * kTile + block / (kTile / 32) * 32;
    const int64_t k0 = tile / p.s.tiles_n * kTile + block % (kTile / 32) * 32;
    if (n0 >= p.w.outputs || k0 >= p.w.x.cols) return;
    const float4* from = reinterpret_cast<const float4*>(p.pieces) +
                         (cut * p.s.pieces * kBlocks + block) * 256 + threadIdx.x;
    await_previous();
    float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 8
    for (int s = 0; s < (int)p.s.pieces; ++s) {
        const float4 a = __ldcg(from + (int64_t)s * (kTile * kTile / 4));
        v.x += a.x; v.y += a.y; v.z += a.z; v.w += a.w;
    }
    // as it was written: threads of a warp hold the 32 rows of four columns
    *reinterpret_cast<float4*>(&turn[threadIdx.x & 31][threadIdx.x / 32 * 4]) = v;
    __syncthreads();
    const int row = threadIdx.x / 8, c = threadIdx.x % 8 * 4;
    v = *reinterpret_cast<const float4*>(&turn[row][c]);
    const int64_t n = n0 + row, k = k0 + c;
    if (n >= p.w.outputs || k >= p.w.x.cols) return;
    const int valid = (int)min((int64_t)4, p.w.x.cols - k);
    const float r[4] = {v.x, v.y, v.z, v.w};
    if (p.w.dw_dtype == kF32)
        put4(r, static_cast<float*>(p.w.dw) + n * p.w.lddw + k, valid, p.vec_out, p.w.accumulate);
    else
        put4(r, static_cast<T*>(p.w.dw) + n * p.w.lddw + k, valid, p.vec_out, p.w.accumulate);
}

// dw without rows: zeros, or left as it is.
template <typename W>
__global__ void clear_kernel(W* dw, int64_t ld, int64_t cols) {
    for (int64_t c = threadIdx.x; c < cols; c += blockDim.x) dw[blockIdx.x * ld + c] = from_f32<W>(0.0f);
}

// Pairs of CTAs that run side by side on the current device (looked up once per device).
int resident_pairs() {
    static std::mutex mutex;
    static int known[64] = {};
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 74;
    std::lock_guard<std::mutex> lock(mutex);
    if (!known[dev]) {
        if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 74;
        known[dev] = sms / 2 > 0 ? sms / 2 : 1;
    }
    return known[dev];
}

Schedule schedule(int64_t rows, int64_t outputs, int64_t cols, int64_t pairs) {
    Schedule s;
    s.tiles_n = (int)((outputs + kTile - 1) / kTile);
    s.tiles_k = (int)((cols + kTile - 1) / kTile);
    s.steps = (rows + kStep - 1) / kStep;
    const int64_t tiles = (int64_t)s.tiles_n * s.tiles_k;
    const int64_t left = tiles % pairs;
    s.pieces = left && s.steps >= kCutSteps ? pairs / left : 1;
    if (s.pieces > 1 && s.pieces > s.steps / kMinSteps) s.pieces = s.steps / kMinSteps;
    s.whole = s.pieces > 1 ? tiles - left : tiles;
    s.units = s.whole + (tiles - s.whole) * s.pieces;
    return s;
}

// The workspace: the pieces' sums, then dy's copy, then the decoded checkpoint.
inline size_t piece_bytes(int64_t rows, int64_t outputs, int64_t cols) {
    const Schedule s = schedule(rows, outputs, cols, resident_pairs());
    return (size_t)(s.units - s.whole) * kTile * kTile * sizeof(float);
}

// cuTensorMapEncodeTiled, through the runtime: the library does not link the driver.
using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                 const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                                 CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                                 CUtensorMapFloatOOBfill);
EncodeTiled encode_tiled() {
    static const EncodeTiled fn = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &found) != cudaSuccess ||
            found != cudaDriverEntryPointSuccess)
            p = nullptr;
        return reinterpret_cast<EncodeTiled>(p);
    }();
    return fn;
}

// Map of a [rows, cols] matrix of 16-bit values in boxes of 64 columns x kStep rows.
template <typename T>
cudaError_t map_columns(CUtensorMap& map, const void* p, int64_t cols, int64_t rows, int64_t pitch) {
    const EncodeTiled encode = encode_tiled();
    if (!encode) return cudaErrorNotSupported;
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)pitch * sizeof(T)};
    const cuuint32_t box[2] = {64, kStep}, unit[2] = {1, 1};
    const CUresult rc = encode(
        &map, std::is_same<T, __half>::value ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16,
        2, const_cast<void*>(p), dims, strides, box, unit, CU_TENSOR_MAP_INTERLEAVE_NONE,
        CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return rc == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

inline int64_t realigned_pitch(int64_t cols) { return (cols + 7) / 8 * 8; }

inline size_t copy_bytes(int64_t rows, int64_t cols) {
    return ((size_t)rows * realigned_pitch(cols) * 2 + 255) / 256 * 256;
}

template <typename T>
cudaError_t launch(const WeightGrad& w, void* workspace, cudaStream_t stream) {
    if (w.rows == 0) {
        if (w.accumulate) return cudaSuccess;
        if (w.dw_dtype == kF32)
            clear_kernel<<<(unsigned)w.outputs, 256, 0, stream>>>(static_cast<float*>(w.dw), w.lddw, w.x.cols);
        else
            clear_kernel<<<(unsigned)w.outputs, 256, 0, stream>>>(static_cast<T*>(w.dw), w.lddw, w.x.cols);
        return cudaGetLastError();
    }
    const int64_t pairs = resident_pairs();
    Params p;
    p.w = w;
    p.s = schedule(w.rows, w.outputs, w.x.cols, pairs);
    p.vec_out = rows_aligned(w.dw, w.lddw, type_size(w.dw_dtype));
    p.pieces = static_cast<float*>(workspace);

    unsigned char* at = static_cast<unsigned char*>(workspace) + piece_bytes(w.rows, w.outputs, w.x.cols);
    // TMA wants rows on 16-byte boundaries: a dy without is copied while the checkpoint is decoded
    const void* dy = w.dy;
    int64_t pitch = w.lddy;
    Realigned copy;
    if (!rows_aligned(w.dy, w.lddy, sizeof(T))) {
        pitch = realigned_pitch(w.outputs);
        copy.from = w.dy;
        copy.ld = w.lddy;
        copy.to = at;
        copy.pitch = pitch;
        copy.cols = w.outputs;
        copy.rows = w.rows;
        dy = at;
        at += copy_bytes(w.rows, w.outputs);
    }
    CUtensorMap map, xmap;
    if (cudaError_t e = map_columns<T>(map, dy, w.outputs, w.rows, pitch)) return e;
    const int64_t xpitch = realigned_pitch(w.x.cols);
    if (cudaError_t e = launch_act8_decode(w.x, at, w.dtype, xpitch, stream, copy)) return e;
    if (cudaError_t e = map_columns<T>(xmap, at, w.x.cols, w.rows, xpitch)) return e;
    if (cudaError_t e = cudaFuncSetAttribute(weight_grad_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                             (int)kSmemBytes))
        return e;
    const int64_t ctas = 2 * (p.s.units < pairs ? p.s.units : pairs);
    if (cudaError_t e = launch_dependent(weight_grad_kernel<T>, dim3((unsigned)ctas), dim3(kThreads), kSmemBytes,
                                         stream, map, xmap, p))
        return e;
    const int64_t cut = (int64_t)p.s.tiles_n * p.s.tiles_k - p.s.whole;
    if (!cut) return cudaSuccess;
    return launch_dependent(weight_grad_pieces_kernel<T>, dim3((unsigned)(cut * (kTile / 32) * (kTile / 32))), dim3(256), 0,
                            stream, p);
}

}  // namespace

size_t weight_grad_workspace(int64_t rows, int64_t outputs, int64_t cols, bool aligned) {
    return piece_bytes(rows, outputs, cols) + (aligned ? 0 : copy_bytes(rows, outputs)) +
           copy_bytes(rows, cols);
}

cudaError_t launch_weight_grad(const WeightGrad& w, void* workspace, cudaStream_t stream) {
    return w.dtype == kBf16 ? launch<__nv_bfloat16>(w, workspace, stream) : launch<__half>(w, workspace, stream);
}

int take_weight_grad_timeout_flag() {
    int v = 0;
    const int zero = 0;
    if (cudaMemcpyFromSymbol(&v, g_weight_grad_timeout, sizeof(v)) != cudaSuccess) return -1;
    if (v && cudaMemcpyToSymbol(g_weight_grad_timeout, &zero, sizeof(zero)) != cudaSuccess) return -1;
    return v;
}

}  // namespace pwlq

// The tensor-core kernel behind the gated feed-forward operators: C = sum over terms of A_s B_s^T, many tokens.
//
// Two blocks of a cluster share a tile of 256 x 256 accumulators: each holds 128 rows of A and 128 of B in shared memory, and
// the pair's first block issues the matrix instructions for both (half the operand traffic of single blocks with 128 x 256
// tiles).  Operands come by tensor-map copies in 128-byte rows of K, six stages ahead; the accumulators of two tiles
// alternate in tensor memory, so that eight warps store one tile while the next one is multiplied.  Blocks walk over tiles.
//
// What bounds it: the tensor pipe, then the GPU's power limit.  8192 x 4096 x 11008 forward takes 1.03 ms in a short run
// (1440 TFLOP/s) and 1.10 ms in a sustained one (1340 TFLOP/s: the pipe is 87 % busy and the clock is down to 1.28 GHz; a
// library product of the same operands sustains 1400).  With e4m3 operands the copies bound it: a stage is multiplied in 256
// clocks, in which a pair wants 64 KiB from L2 (4095 x 4096 x 11008: 0.31 ms, the copies alone 0.21 ms).
#pragma once
#include "ops_common.cuh"
#include "umma.cuh"

namespace collage {
namespace ops {

constexpr float kGeluC = 0.7978845608028654f;      // sqrt(2 / pi)
constexpr float kGeluD = 0.044715f;

// tanh's argument for GELU.  Beyond |g| = 16 the tanh is 1 to the last bit: the clamp keeps g^3 and the slope's factors
// finite.  A NaN passes.
__device__ __forceinline__ float gelu_inner(float g) {
    const float c = g > 16.0f ? 16.0f : g < -16.0f ? -16.0f : g;
    return kGeluC * __fmaf_rn(kGeluD * c * c, c, c);
}
// 1 / (1 + exp(-v)); GELU's (1 + tanh(w)) / 2 is the same function of 2 w.  The fast exponential is off by up to 2 + 1.2 |v| units of
// its last place, which for negative v is the result's relative error: 6e-6 at -40, 1.2e-5 at -87.  Below v = -87.3 the
// denominator passes 2^126 and the fast quotient is 0, where the function is at most 1.2e-38.  Neither shows in bfloat16 results, which
// are rounded by 2^-9 of their value (g times the function is below 1.1e-36 there).
__device__ __forceinline__ float logistic(float v) { return __fdividef(1.0f, 1.0f + __expf(-v)); }

__device__ __forceinline__ float activate(int kind, float g) {
    return g * logistic(kind == COLLAGE_ACT_SILU ? g : 2.0f * gelu_inner(g));
}
// a(g) and a'(g)
__device__ __forceinline__ float2 activate_and_slope(int kind, float g) {
    if (kind == COLLAGE_ACT_SILU) {
        const float s = logistic(g);
        return make_float2(g * s, s * __fmaf_rn(g, 1.0f - s, 1.0f));
    }
    const float c = g > 16.0f ? 16.0f : g < -16.0f ? -16.0f : g;
    const float s = logistic(2.0f * gelu_inner(g));
    return make_float2(g * s, __fmaf_rn(2.0f * c * s * (1.0f - s), kGeluC * __fmaf_rn(3.0f * kGeluD * c, c, 1.0f), s));
}

// Code of the first bounded wait of this kernel that gave up (collage_pipeline_fault reports it).
static __device__ unsigned int g_product_fault;

// One launch: `problems` outputs of m x n (they share b when there are two), each a sum of `terms` products over k.
// GATED: one problem, one term, b[0] and b[1] the two weights of out[0] = h (out[1], out[2] = gate, up if kept).
struct TileArgs {
    CUtensorMap a[2], b[2], out[3];
    const float* a_scale;
    const float* b_scale[2];
    uint32_t m, n;                       // of the output
    uint32_t m_tiles, n_tiles, group;    // tiles are taken `group` rows of tiles at a time
    uint32_t problems, terms, k_blocks;  // k_blocks: of one term
    int keep, activation;
};

constexpr int kOperandBytes = 128 * umma::kRowBytes;          // 128 indexes x 128 bytes of K: 16 KiB
constexpr int kStageBytes = 2 * kOperandBytes;
constexpr int kStages = 6;
constexpr int kUnitCols = 32;                                 // columns of one output store, 64 bytes, of a warp's 32 rows
constexpr int kUnitBytes = 32 * 2 * kUnitCols;
constexpr int kUnits = 2;                                     // of each storing warp
constexpr int kStoreWarps = 8;
constexpr int kTileThreads = 128 + 32 * kStoreWarps;          // warp 0 loads, 1 multiplies, 2 owns tensor memory, 4-11 store
constexpr int kTileSmem = 1024 + kStages * kStageBytes + kStoreWarps * kUnits * kUnitBytes + 256;

struct TileBarriers {
    uint64_t full[kStages], empty[kStages], done[2], drained[2];
    uint32_t tmem;
};
static_assert(sizeof(TileBarriers) <= 256, "barriers fit their place");

struct TilePlace {
    uint32_t problem, m, n;              // tile indexes
};
__device__ __forceinline__ TilePlace place_of(const TileArgs& p, uint32_t tile) {
    const uint32_t per = p.m_tiles * p.n_tiles, problem = tile / per, t = tile % per;
    const uint32_t in_group = p.group * p.n_tiles, g = t / in_group, r = t % in_group;
    const uint32_t rows = min(p.group, p.m_tiles - g * p.group);
    return {problem, g * p.group + r % rows, r / rows};
}

// A_MN: A is stored with its rows' index contiguous (a transposed operand); B is, where the kernel is not GATED.
template <bool E4M3, bool A_MN, bool GATED>
__global__ void __launch_bounds__(kTileThreads, 1) tile_kernel(const __grid_constant__ TileArgs p) {
    constexpr bool B_MN = !GATED;
    constexpr uint32_t CTAS = 2, kN = 128 * CTAS;             // blocks of a tile, accumulator columns
    constexpr uint32_t kOut = GATED ? kN / 2 : kN;            // output columns of a tile
    constexpr uint32_t kK = E4M3 ? 128 : 64;                  // K elements in 128 bytes
    constexpr uint32_t kIdesc = umma::instr_desc(E4M3 ? 0 : 1, A_MN, B_MN, 128 * CTAS, kN);
    extern __shared__ uint8_t raw_smem[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw_smem) + 1023) & ~static_cast<uintptr_t>(1023));
    uint8_t* staging = smem + kStages * kStageBytes;
    TileBarriers* bars = reinterpret_cast<TileBarriers*>(staging + kStoreWarps * kUnits * kUnitBytes);
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = umma::cluster_rank();
    const uint32_t tiles = p.problems * p.m_tiles * p.n_tiles, first = blockIdx.x / CTAS, step = gridDim.x / CTAS;
    const uint32_t blocks = p.terms * p.k_blocks;

    if (threadIdx.x == 0) {
        for (int i = 0; i < kStages; ++i) {
            pipe::mbar_init(&bars->full[i], 1);
            pipe::mbar_init(&bars->empty[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            pipe::mbar_init(&bars->done[i], 1);
            pipe::mbar_init(&bars->drained[i], kStoreWarps * CTAS);
        }
        pipe::mbar_init_fence();
        for (int i = 0; i < 2; ++i) {
            umma::prefetch_map(&p.a[i]);
            umma::prefetch_map(&p.b[i]);
        }
    }
    if (warp == 2) umma::tmem_alloc<CTAS>(&bars->tmem, 2 * kN);
    umma::fence_before();
    __syncthreads();
    umma::cluster_sync();                                     // the other block's barriers exist
    umma::fence_after();
    after_previous();
    const uint32_t tmem = bars->tmem;

    // The first two warps run their loops as a whole, so that addresses and descriptors stay in uniform registers, and one
    // thread issues.  (With the loops under `lane == 0` the tensor pipe was busy 65 % of the time instead of 87 %.)
    if (warp == 0) {
        uint32_t stage = 0, phase = 0, used = 0;
        bool ok = true;
        for (uint32_t tile = first; tile < tiles && ok; tile += step) {
            const TilePlace at = place_of(p, tile);
            const int m0 = static_cast<int>(at.m * 128 * CTAS + rank * 128), n0 = static_cast<int>(at.n * kOut);
            for (uint32_t kb = 0; kb < blocks; ++kb) {
                if (!(ok = umma::warp_wait(&bars->empty[stage], phase ^ 1, 200, &g_product_fault))) break;
                if (umma::elected()) {
                    if (rank == 0) pipe::mbar_arrive_expect_tx(&bars->full[stage], kStageBytes * CTAS);
                    const uint32_t bar = umma::cluster_addr(&bars->full[stage], 0);
                    uint8_t *sa = smem + stage * kStageBytes, *sb = sa + kOperandBytes;
                    const uint32_t term = kb / p.k_blocks;
                    const int k = static_cast<int>((kb - term * p.k_blocks) * kK);
                    const CUtensorMap* a = &p.a[p.problems > 1 ? at.problem : term];
                    if constexpr (A_MN) {
                        umma::tile_load<CTAS>(sa, a, m0, k, bar);
                        umma::tile_load<CTAS>(sa + kOperandBytes / 2, a, m0 + 64, k, bar);
                    } else {
                        umma::tile_load<CTAS>(sa, a, k, m0, bar);
                    }
                    if constexpr (GATED) {                    // the first block's columns are gates, the second one's ups
                        umma::tile_load<CTAS>(sb, &p.b[rank], k, n0, bar);
                    } else {
                        const int n = n0 + static_cast<int>(rank * 128);
                        umma::tile_load<CTAS>(sb, &p.b[term], n, k, bar);
                        umma::tile_load<CTAS>(sb + kOperandBytes / 2, &p.b[term], n + 64, k, bar);
                    }
                }
                __syncwarp();
                used = min(used + 1, static_cast<uint32_t>(kStages));
                if (++stage == kStages) { stage = 0; phase ^= 1; }
            }
        }
        // The last uses of the stages: nothing arrives in this block any more once they are over.  After a wait that was given up
        // they may never be; then the copies themselves are waited for: both blocks' by the first block, on whose barriers they are
        // counted, and a millisecond by the second, for what it has sent for beyond those.
        for (uint32_t i = 0; i < used; ++i) {
            stage = stage ? stage - 1 : kStages - 1;
            if (stage == kStages - 1) phase ^= 1;
            if (ok) ok = umma::warp_wait(&bars->empty[stage], phase, 201, &g_product_fault);
            if (!ok && rank == 0) umma::warp_wait(&bars->full[stage], phase, 206, &g_product_fault);
        }
        if (!ok && rank == 1)
            for (const unsigned long long t0 = pipe::global_ns(); pipe::global_ns() - t0 < 1000000;) {}
    } else if (warp == 1) {
        uint32_t stage = 0, phase = 0, n_tile = 0, committed = 0;
        bool ok = rank == 0;
        const uint32_t smem0 = umma::smem_addr(smem);
        for (uint32_t tile = first; tile < tiles && ok; tile += step, ++n_tile) {
            const uint32_t acc = n_tile & 1;
            if (!(ok = umma::warp_wait(&bars->drained[acc], ((n_tile >> 1) & 1) ^ 1, 202, &g_product_fault))) break;
            umma::fence_after();
            const uint32_t d = tmem + acc * kN;
            for (uint32_t kb = 0; kb < blocks; ++kb) {
                if (!(ok = umma::warp_wait(&bars->full[stage], phase, 203, &g_product_fault))) {
                    if (umma::elected()) umma::commit<CTAS>(&bars->done[acc]);      // of what has been issued
                    break;
                }
                umma::fence_after();
                const uint32_t sa = smem0 + stage * kStageBytes, sb = sa + kOperandBytes;
                const uint64_t da = umma::operand_desc(sa, A_MN ? kOperandBytes / 2 : 16, 1024);
                const uint64_t db = umma::operand_desc(sb, B_MN ? kOperandBytes / 2 : 16, 1024);
                if (umma::elected()) {
                    // one instruction takes 32 bytes of K: 32 bytes along the rows, or 16 rows of 128 bytes
#pragma unroll
                    for (uint32_t i = 0; i < 4; ++i)
                        umma::mma<CTAS, E4M3>(d, da + i * (A_MN ? 2048 : 32) / 16, db + i * (B_MN ? 2048 : 32) / 16, kIdesc, kb > 0 || i > 0);
                    umma::commit<CTAS>(&bars->empty[stage]);
                    if (kb + 1 == blocks) umma::commit<CTAS>(&bars->done[acc]);
                }
                __syncwarp();
                if (++stage == kStages) { stage = 0; phase ^= 1; }
            }
            ++committed;
        }
        // no matrix instruction is under way when operands and accumulators are given up
        if (committed) umma::warp_wait(&bars->done[(committed - 1) & 1], ((committed - 1) >> 1) & 1, 205, &g_product_fault);
    } else if (warp >= 4) {
        // Two warps for each quarter of the rows (the quarter of tensor memory that a warp can read is its number's), each
        // with half of the columns.  A warp stages and stores its 32 rows by itself.
        const uint32_t quarter = warp & 3, half = (warp - 4) >> 2;
        const uint32_t lane_base = tmem + (quarter << 21), c_begin = half * (kOut / 2), c_end = c_begin + kOut / 2;
        uint8_t* slots = staging + (warp - 4) * kUnits * kUnitBytes;
        uint32_t unit = 0, n_tile = 0;
        // 32 columns of this thread's row, as 16 words, through shared memory to the output
        auto store_unit = [&](const CUtensorMap* map, int x, int y, const uint32_t (&w)[16]) {
            uint8_t* slot = slots + (unit % kUnits) * kUnitBytes;
            if (lane == 0) asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(kUnits - 1) : "memory");
            __syncwarp();
            uint4* line = reinterpret_cast<uint4*>(slot + lane * 64);
#pragma unroll
            for (int c = 0; c < 4; ++c) line[c ^ ((lane >> 1) & 3)] = make_uint4(w[4 * c], w[4 * c + 1], w[4 * c + 2], w[4 * c + 3]);
            pipe::fence_async_smem();
            __syncwarp();
            if (lane == 0) {
                if (y < static_cast<int>(p.m)) umma::tile_store(map, x, y, slot);
                pipe::bulk_commit();
            }
            ++unit;
        };
        auto packed = [](const float (&v)[32], uint32_t (&w)[16]) {
#pragma unroll
            for (int i = 0; i < 16; ++i) w[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
        };
        for (uint32_t tile = first; tile < tiles; tile += step, ++n_tile) {
            const uint32_t acc = n_tile & 1;
            if (!umma::warp_wait(&bars->done[acc], (n_tile >> 1) & 1, 204, &g_product_fault)) break;
            umma::fence_after();
            const TilePlace at = place_of(p, tile);
            const int m0 = static_cast<int>(at.m * 128 * CTAS + rank * 128 + quarter * 32);
            const uint32_t n0 = at.n * kOut;
            const uint32_t cols = min(kOut, p.n - n0);
            float row_scale = 0.0f;
            if constexpr (E4M3)
                if (m0 + lane < p.m) row_scale = p.a_scale[m0 + lane];
            uint32_t w[16];
#pragma unroll 1
            for (uint32_t c = c_begin; c < c_end; c += kUnitCols) {
                float v[32];
                umma::tmem_load32(lane_base + acc * kN + c, v);
                if constexpr (GATED) {
                    float u[32];
                    umma::tmem_load32(lane_base + acc * kN + kOut + c, u);
                    umma::tmem_wait(v);
                    umma::tmem_wait(u);
                    if (c + kUnitCols == c_end) {             // the accumulators are read: they may be overwritten
                        umma::fence_before();
                        __syncwarp();
                        if (lane == 0) umma::cluster_arrive(umma::cluster_addr(&bars->drained[acc], 0));
                    }
                    if (c >= cols) continue;
                    if constexpr (E4M3) {
#pragma unroll
                        for (int i = 0; i < 32; ++i) {
                            const uint32_t n = min(n0 + c + i, p.n - 1);
                            v[i] *= row_scale * __ldg(p.b_scale[0] + n);
                            u[i] *= row_scale * __ldg(p.b_scale[1] + n);
                        }
                    }
                    if (p.keep) {
                        packed(v, w);
                        store_unit(&p.out[1], static_cast<int>(n0 + c), m0, w);
                        packed(u, w);
                        store_unit(&p.out[2], static_cast<int>(n0 + c), m0, w);
                    }
#pragma unroll
                    for (int i = 0; i < 32; ++i) v[i] = activate(p.activation, v[i]) * u[i];
                    packed(v, w);
                    store_unit(&p.out[0], static_cast<int>(n0 + c), m0, w);
                } else {
                    umma::tmem_wait(v);
                    if (c + kUnitCols == c_end) {
                        umma::fence_before();
                        __syncwarp();
                        if (lane == 0) umma::cluster_arrive(umma::cluster_addr(&bars->drained[acc], 0));
                    }
                    if (c >= cols) continue;
                    packed(v, w);
                    store_unit(&p.out[at.problem], static_cast<int>(n0 + c), m0, w);
                }
            }
        }
        if (lane == 0) pipe::bulk_wait_all();
    }
    __syncwarp();
    umma::fence_before();
    __syncthreads();
    umma::cluster_sync();                                     // both blocks are done with each other's memory
    umma::fence_after();
    if (warp == 2) umma::tmem_free<CTAS>(tmem, 2 * kN);
}

}  // namespace ops
}  // namespace collage

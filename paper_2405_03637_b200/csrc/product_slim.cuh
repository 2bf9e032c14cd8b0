// The products of few tokens: weights as the 128 rows of a tile, tokens as its 16 to 128 columns, the sum over K split over
// a cluster.
//
// Such a product reads each weight once and multiplies it with few tokens: the bytes of the weights bound it, and what
// matters is that every SM has copies under way all the time.  So a tile takes all 128 rows of the matrix instruction from
// the weights, two or three blocks share an SM, and where there are fewer tiles than SMs the blocks of a cluster take parts of K
// and join their sums through each other's shared memory, in the order of K.  One token x 4096 x 11008 (180 MB of weights):
// 31.7 us, 5.7 TB/s; 16 tokens with e4m3 weights (90 MB): 19 us, 4.8 TB/s; dx of 16 tokens 35 us.
#pragma once
#include "product_tile.cuh"

namespace collage {
namespace ops {

// out[t, i] for tokens t < n and weight indexes i < m.  GATED: a[0] and a[1] are the two weights, 64 indexes of each in a
// tile, out[0] = h (out[1], out[2] = gate, up if kept).  Otherwise the sum over `terms` of A_s B_s^T, 128 indexes a tile.
struct SlimArgs {
    CUtensorMap a[2], b[2];
    const float* row_scale[2];           // of the weights (e4m3)
    const float* token_scale;
    uint16_t* out[3];
    uint64_t ldo[3];
    uint32_t m, n, token_tiles, k_blocks, terms, split, stages;
    int keep, activation;
};

constexpr int kSlimThreads = 128;

template <int NT>
__host__ __device__ constexpr int slim_stage_bytes() { return kOperandBytes + NT * static_cast<int>(umma::kRowBytes); }
// Stages (the sums over the tile take their place afterwards): as many as leave room for two blocks on an SM, three of the
// narrowest (33 against 36 us for one token x 4096 x 11008), or all that fit where there is at most one block for an SM.
constexpr int kMaxSlimStages = 10;
template <int NT>
__host__ __device__ constexpr int slim_stages(bool alone) {
    return alone ? 212 * 1024 / slim_stage_bytes<NT>() : NT <= 16 ? 4 : NT <= 32 ? 5 : NT <= 64 ? 4 : 3;
}
template <int NT>
constexpr int slim_smem(bool alone) { return 1024 + (slim_stages<NT>(alone) > kMaxSlimStages ? kMaxSlimStages : slim_stages<NT>(alone)) * slim_stage_bytes<NT>(); }

// The end of a slim tile, by all threads of the block: its accumulators to shared memory, the cluster's parts joined in the
// order of K, the results stored (a sum of products in out[which]).  VECTORS: whole vectors fit the outputs.
template <bool E4M3, bool GATED, int NT, bool VECTORS, typename Args>
__device__ __forceinline__ void finish_slim_tile(const Args& p, uint8_t* smem, uint32_t tmem, uint32_t rank, uint32_t t0, uint32_t i0, uint32_t which = 0) {
    __syncthreads();                                 // the sums are complete and the stages free
    umma::fence_after();
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    float* sums = reinterpret_cast<float*>(smem);    // [NT][128]: a token's 128 indexes
    const uint32_t row = threadIdx.x;
#pragma unroll 1
    for (uint32_t c = 0; c < NT && warp < 4; c += 16) {
        float v[16];
        umma::tmem_load16(tmem + (warp << 21) + c, v);
        umma::tmem_wait(v);
#pragma unroll
        for (uint32_t i = 0; i < 16; ++i) sums[(c + i) * 128 + row] = v[i];
    }
    umma::fence_before();
    if (p.split > 1) umma::cluster_sync();
    else __syncthreads();
    umma::fence_after();
    if (warp == 2) umma::tmem_free<1>(tmem, NT < 32 ? 32 : NT);

    // Tokens over the cluster's blocks and their warps, four at a time; parts of the sum in the order of K.
    const uint32_t tokens = min(static_cast<uint32_t>(NT), p.n - t0);
    auto store2 = [&](uint16_t* at, uint32_t i, float a, float b) {     // indexes i and i + 1
        if constexpr (VECTORS) {                     // m is a multiple of 8, rows begin on 16 bytes
            *reinterpret_cast<uint32_t*>(at) = pack_bf16(a, b);
        } else {
            at[0] = to_bf16(a);
            if (i + 1 < p.m) at[1] = to_bf16(b);
        }
    };
    auto part = [&](uint32_t r, uint32_t t, uint32_t i) {               // four floats of block r's sums
        float4 q;
        if (p.split == 1) return *reinterpret_cast<const float4*>(sums + t * 128 + i);
        asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(q.x), "=f"(q.y), "=f"(q.z), "=f"(q.w) : "r"(umma::cluster_addr(sums + t * 128 + i, r)));
        return q;
    };
    for (uint32_t first = rank * 16 + warp * 4; first < tokens && warp < 4; first += p.split * 16) {
        float4 v[4] = {};
        for (uint32_t r = 0; r < p.split; ++r) {
            float4 q[4];
#pragma unroll
            for (uint32_t e = 0; e < 4; ++e) q[e] = part(r, first + e, 4 * lane);      // NT is a multiple of 4
#pragma unroll
            for (uint32_t e = 0; e < 4; ++e) { v[e].x += q[e].x; v[e].y += q[e].y; v[e].z += q[e].z; v[e].w += q[e].w; }
        }
        if constexpr (GATED) {
            // lanes 0-15 have four gates each, lanes 16-31 the ups that belong to them: the lower two of four to the lower lane
            const bool low = lane < 16;
            const uint32_t i = i0 + 4 * (lane & 15) + (low ? 0 : 2);
            float2 row_g = {1.0f, 1.0f}, row_u = {1.0f, 1.0f};
            if constexpr (E4M3)
                if (i < p.m) {
                    const uint32_t n = min(i + 1, p.m - 1);
                    row_g = make_float2(p.row_scale[0][i], p.row_scale[0][n]);
                    row_u = make_float2(p.row_scale[1][i], p.row_scale[1][n]);
                }
#pragma unroll
            for (uint32_t e = 0; e < 4; ++e) {
                const float a = __shfl_xor_sync(0xFFFFFFFFu, low ? v[e].z : v[e].x, 16), b = __shfl_xor_sync(0xFFFFFFFFu, low ? v[e].w : v[e].y, 16);
                float2 g = low ? make_float2(v[e].x, v[e].y) : make_float2(a, b), u = low ? make_float2(a, b) : make_float2(v[e].z, v[e].w);
                if (first + e >= tokens || i >= p.m) continue;
                const uint64_t token = t0 + first + e;
                if constexpr (E4M3) {
                    const float s = p.token_scale[token];
                    g.x *= s * row_g.x; g.y *= s * row_g.y;
                    u.x *= s * row_u.x; u.y *= s * row_u.y;
                }
                if (p.keep) {
                    store2(p.out[1] + token * p.ldo[1] + i, i, g.x, g.y);
                    store2(p.out[2] + token * p.ldo[2] + i, i, u.x, u.y);
                }
                store2(p.out[0] + token * p.ldo[0] + i, i, activate(p.activation, g.x) * u.x, activate(p.activation, g.y) * u.y);
            }
        } else {
            const uint32_t i = i0 + 4 * lane;
#pragma unroll
            for (uint32_t e = 0; e < 4; ++e)
                if (first + e < tokens && i < p.m) {
                    uint16_t* at = p.out[which] + (t0 + first + e) * p.ldo[which] + i;
                    if constexpr (VECTORS) {
                        *reinterpret_cast<uint2*>(at) = make_uint2(pack_bf16(v[e].x, v[e].y), pack_bf16(v[e].z, v[e].w));
                    } else {
                        store2(at, i, v[e].x, v[e].y);
                        if (i + 2 < p.m) store2(at + 2, i + 2, v[e].z, v[e].w);
                    }
                }
        }
    }
    if (p.split > 1) umma::cluster_sync_any();       // no block leaves while another reads its sums
}

// One tile by one block (`rank` of its cluster's `split`).  A_MN, B_MN: the operand is stored with its index contiguous.
template <bool E4M3, bool A_MN, bool B_MN, bool GATED, int NT>
__device__ __forceinline__ void slim_tile(const SlimArgs& p, uint32_t tile, uint32_t rank) {
    constexpr uint32_t kBytes = slim_stage_bytes<NT>();
    constexpr uint32_t kK = E4M3 ? 128 : 64, kIndexes = GATED ? 64 : 128;
    constexpr uint32_t kIdesc = umma::instr_desc(E4M3 ? 0 : 1, A_MN, B_MN, 128, NT);
    static_assert(slim_stages<NT>(false) * kBytes >= NT * 512, "the tile's sums fit the stages");
    const uint32_t stages = p.stages;
    extern __shared__ uint8_t raw_smem[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw_smem) + 1023) & ~static_cast<uintptr_t>(1023));
    __shared__ uint64_t full[kMaxSlimStages], empty[kMaxSlimStages], done;
    __shared__ uint32_t tmem_slot, lost;             // lost: a wait was given up
    const uint32_t warp = threadIdx.x >> 5;
    static_assert(!B_MN || NT % 64 == 0, "an operand stored by its index comes in boxes of 64 indexes");
    // with several outputs (B_MN) the tiles of the first come first
    const uint32_t per = p.token_tiles * ((p.m + kIndexes - 1) / kIndexes), which = B_MN ? tile / per : 0, place = B_MN ? tile % per : tile;
    const uint32_t t0 = place % p.token_tiles * NT, i0 = place / p.token_tiles * kIndexes;
    const uint32_t blocks = p.terms * p.k_blocks;
    const uint32_t begin = static_cast<uint32_t>(static_cast<uint64_t>(blocks) * rank / p.split);
    const uint32_t end = static_cast<uint32_t>(static_cast<uint64_t>(blocks) * (rank + 1) / p.split);

    if (threadIdx.x == 0) {
        for (uint32_t i = 0; i < stages; ++i) {
            pipe::mbar_init(&full[i], 1);
            pipe::mbar_init(&empty[i], 1);
        }
        pipe::mbar_init(&done, 1);
        pipe::mbar_init_fence();
        lost = 0;
    }
    if (warp == 2) umma::tmem_alloc<1>(&tmem_slot, NT < 32 ? 32 : NT);
    umma::fence_before();
    __syncthreads();
    umma::fence_after();
    after_previous();
    const uint32_t tmem = tmem_slot;

    uint32_t stage = 0, phase = 0, kb = begin;
    if (warp == 0) {
        for (; kb < end; ++kb) {
            if (!umma::warp_wait(&empty[stage], phase ^ 1, 210, &g_product_fault)) {
                lost = 1;
                break;
            }
            if (umma::elected()) {
                pipe::mbar_arrive_expect_tx(&full[stage], kBytes);
                const uint32_t bar = umma::smem_addr(&full[stage]);
                uint8_t *sa = smem + stage * kBytes, *sb = sa + kOperandBytes;
                const uint32_t term = kb / p.k_blocks;
                const int k = static_cast<int>((kb - term * p.k_blocks) * kK);
                if constexpr (GATED) {
                    umma::tile_load<1>(sa, &p.a[0], k, static_cast<int>(i0), bar);
                    umma::tile_load<1>(sa + kOperandBytes / 2, &p.a[1], k, static_cast<int>(i0), bar);
                } else if constexpr (A_MN) {
                    umma::tile_load<1>(sa, &p.a[term], static_cast<int>(i0), k, bar);
                    umma::tile_load<1>(sa + kOperandBytes / 2, &p.a[term], static_cast<int>(i0) + 64, k, bar);
                }
                if constexpr (B_MN) {
#pragma unroll
                    for (int n = 0; n < NT / 64; ++n) umma::tile_load<1>(sb + n * (kOperandBytes / 2), &p.b[which], static_cast<int>(t0) + 64 * n, k, bar);
                } else {
                    umma::tile_load<1>(sb, &p.b[term], k, static_cast<int>(t0), bar);
                }
            }
            __syncwarp();
            if (++stage == stages) { stage = 0; phase ^= 1; }
        }
    } else if (warp == 1) {
        const uint32_t smem0 = umma::smem_addr(smem);
        bool ok = true;
        for (; kb < end; ++kb) {
            if (!(ok = umma::warp_wait(&full[stage], phase, 211, &g_product_fault))) break;
            umma::fence_after();
            const uint32_t sa = smem0 + stage * kBytes;
            const uint64_t da = umma::operand_desc(sa, A_MN ? kOperandBytes / 2 : 16, 1024), db = umma::operand_desc(sa + kOperandBytes, B_MN ? kOperandBytes / 2 : 16, 1024);
            if (umma::elected()) {
#pragma unroll
                for (uint32_t i = 0; i < 4; ++i)
                    umma::mma<1, E4M3>(tmem, da + i * (A_MN ? 2048 : 32) / 16, db + i * (B_MN ? 2048 : 32) / 16, kIdesc, kb > begin || i > 0);
                umma::commit<1>(&empty[stage]);
                if (kb + 1 == end) umma::commit<1>(&done);
            }
            __syncwarp();
            if (++stage == stages) { stage = 0; phase ^= 1; }
        }
        if (!ok && umma::elected()) umma::commit<1>(&done);        // of what has been issued
        if (!umma::warp_wait(&done, 0, 212, &g_product_fault) || !ok) lost = 1;
    }
    finish_slim_tile<E4M3, GATED, NT, true>(p, smem, tmem, rank, t0, i0, which);
    // Where a wait was given up, copies may still be under way that nobody has waited for, the last uses of the stages: the block
    // stays until they have come.
    if (warp == 0 && lost)
        for (uint32_t used = min(kb - begin, stages); used > 0; --used) {
            stage = stage ? stage - 1 : stages - 1;
            if (stage == stages - 1) phase ^= 1;
            umma::warp_wait(&full[stage], phase, 213, &g_product_fault);
        }
}

template <bool E4M3, bool A_MN, bool GATED, int NT>
__global__ void __launch_bounds__(kSlimThreads) slim_kernel(const __grid_constant__ SlimArgs p) {
    slim_tile<E4M3, A_MN, false, GATED, NT>(p, blockIdx.x / p.split, p.split > 1 ? umma::cluster_rank() : 0);
}

// The gradients of small layers in one launch: the first blocks make dx = dgate w_gate + dup w_up, the others, which need not
// wait for them, tiles of dw_gate = dgate^T x and dw_up = dup^T x (tokens are K there, ffn takes the tokens' place).
template <int NT>
__global__ void __launch_bounds__(kSlimThreads) slim_backward_kernel(const __grid_constant__ SlimArgs dx, const __grid_constant__ SlimArgs dw, uint32_t dx_blocks,
                                                                     uint32_t dw_tiles) {
    if (blockIdx.x < dx_blocks)
        slim_tile<false, true, false, false, NT>(dx, blockIdx.x / dx.split, dx.split > 1 ? umma::cluster_rank() : 0);
    else if (blockIdx.x - dx_blocks < dw_tiles)
        slim_tile<false, true, true, false, 128>(dw, blockIdx.x - dx_blocks, 0);
}

}  // namespace ops
}  // namespace collage

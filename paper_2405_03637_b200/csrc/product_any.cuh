// The products of matrices that tensor maps cannot describe (rows that do not begin on 16 bytes, odd widths): slim tiles
// whose operands eight warps bring to shared memory element by element, in the layout that a tile load would have made.
// The element loads bound it (4096 x 4097 x 11009 forward: 5.0 ms, 150 TFLOP/s); sums are held in float as elsewhere.
#pragma once
#include "product_slim.cuh"

namespace collage {
namespace ops {

// An operand of a product, element (i, k) at data + i * row + k * col; one of the two strides is 1.
struct Operand {
    const void* data;
    uint64_t row, col;
};

// As SlimArgs: out[t, i] = sum over terms and k of a[i, k] b[t, k].
struct AnyArgs {
    Operand a[2], b[2];
    const float* row_scale[2];
    const float* token_scale;
    uint16_t* out[3];
    uint64_t ldo[3];
    uint32_t m, n, k, token_tiles, k_blocks, terms, split;
    int keep, activation;
};

constexpr int kAnyLoaders = 256, kAnyThreads = 128 + kAnyLoaders, kAnyStages = 3;
template <int NT>
constexpr int any_smem() { return 1024 + kAnyStages * slim_stage_bytes<NT>(); }

// `rows` rows of 128 bytes of K (from k0) into the swizzled tile at dst: row r holds index first + r of the operand, zeros from
// `limit` on and from K's end on.  Threads are laid along the operand's contiguous direction.
template <typename T>
__device__ __forceinline__ void bring(const Operand& o, uint8_t* dst, uint32_t rows, uint64_t first, uint64_t limit, uint64_t k0, uint64_t k_end, uint32_t t) {
    constexpr uint32_t kPer = 16 / sizeof(T), kAhead = 2;
    const T* data = static_cast<const T*>(o.data);
    const uint32_t tasks = rows * 8;                          // 16 bytes each
    for (uint32_t q0 = t; q0 < tasks; q0 += kAnyLoaders * kAhead) {
        union { uint4 q; T e[kPer]; } v[kAhead];
        uint32_t place[kAhead];
#pragma unroll
        for (uint32_t n = 0; n < kAhead; ++n) {
            const uint32_t q = q0 + n * kAnyLoaders, r = o.col == 1 ? q >> 3 : q % rows, c = o.col == 1 ? q & 7 : q / rows;
            const uint64_t i = first + r, k = k0 + c * kPer;
            place[n] = r * umma::kRowBytes + ((c ^ (r & 7)) << 4);
            v[n].q = make_uint4(0, 0, 0, 0);
            if (q < tasks && i < limit) {
                const T* at = data + i * o.row + k * o.col;
                if (k + kPer <= k_end) {
#pragma unroll
                    for (uint32_t e = 0; e < kPer; ++e) v[n].e[e] = at[e * o.col];
                } else {
#pragma unroll
                    for (uint32_t e = 0; e < kPer; ++e)
                        if (k + e < k_end) v[n].e[e] = at[e * o.col];
                }
            }
        }
#pragma unroll
        for (uint32_t n = 0; n < kAhead; ++n)
            if (q0 + n * kAnyLoaders < tasks) *reinterpret_cast<uint4*>(dst + place[n]) = v[n].q;
    }
}

template <bool E4M3, bool GATED, int NT>
__global__ void __launch_bounds__(kAnyThreads) any_kernel(const __grid_constant__ AnyArgs p) {
    using T = std::conditional_t<E4M3, uint8_t, uint16_t>;
    constexpr uint32_t kBytes = slim_stage_bytes<NT>(), kK = umma::kRowBytes / sizeof(T), kIndexes = GATED ? 64 : 128;
    constexpr uint32_t kIdesc = umma::instr_desc(E4M3 ? 0 : 1, false, false, 128, NT);
    static_assert(kAnyStages * kBytes >= NT * 512, "the tile's sums fit the stages");
    extern __shared__ uint8_t raw_smem[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw_smem) + 1023) & ~static_cast<uintptr_t>(1023));
    __shared__ uint64_t full[kAnyStages], empty[kAnyStages], done;
    __shared__ uint32_t tmem_slot;
    const uint32_t warp = threadIdx.x >> 5;
    const uint32_t rank = p.split > 1 ? umma::cluster_rank() : 0, tile = blockIdx.x / p.split;
    const uint32_t t0 = tile % p.token_tiles * NT, i0 = tile / p.token_tiles * kIndexes;
    const uint32_t blocks = p.terms * p.k_blocks;
    const uint32_t begin = static_cast<uint32_t>(static_cast<uint64_t>(blocks) * rank / p.split);
    const uint32_t end = static_cast<uint32_t>(static_cast<uint64_t>(blocks) * (rank + 1) / p.split);

    if (threadIdx.x == 0) {
        for (uint32_t i = 0; i < kAnyStages; ++i) {
            pipe::mbar_init(&full[i], kAnyLoaders);
            pipe::mbar_init(&empty[i], 1);
        }
        pipe::mbar_init(&done, 1);
        pipe::mbar_init_fence();
    }
    if (warp == 2) umma::tmem_alloc<1>(&tmem_slot, NT < 32 ? 32 : NT);
    umma::fence_before();
    __syncthreads();
    umma::fence_after();
    after_previous();
    const uint32_t tmem = tmem_slot;

    uint32_t stage = 0, phase = 0;
    if (warp >= 4) {
        const uint32_t t = threadIdx.x - 128;
        for (uint32_t kb = begin; kb < end; ++kb) {
            if (!pipe::mbar_wait(&empty[stage], phase ^ 1, 220, &g_product_fault)) break;
            uint8_t *sa = smem + stage * kBytes, *sb = sa + kOperandBytes;
            const uint32_t term = kb / p.k_blocks;
            const uint64_t k0 = static_cast<uint64_t>(kb - term * p.k_blocks) * kK;
            if constexpr (GATED) {
                bring<T>(p.a[0], sa, 64, i0, p.m, k0, p.k, t);
                bring<T>(p.a[1], sa + kOperandBytes / 2, 64, i0, p.m, k0, p.k, t);
            } else {
                bring<T>(p.a[term], sa, 128, i0, p.m, k0, p.k, t);
            }
            bring<T>(p.b[term], sb, NT, t0, p.n, k0, p.k, t);
            pipe::fence_async_smem();                // for the matrix instructions, which read by the asynchronous proxy
            pipe::mbar_arrive(&full[stage]);
            if (++stage == kAnyStages) { stage = 0; phase ^= 1; }
        }
    } else if (warp == 1) {
        const uint32_t smem0 = umma::smem_addr(smem);
        bool ok = true;
        for (uint32_t kb = begin; kb < end; ++kb) {
            if (!(ok = umma::warp_wait(&full[stage], phase, 221, &g_product_fault))) break;
            umma::fence_after();
            const uint32_t sa = smem0 + stage * kBytes;
            const uint64_t da = umma::operand_desc(sa, 16, 1024), db = umma::operand_desc(sa + kOperandBytes, 16, 1024);
            if (umma::elected()) {
#pragma unroll
                for (uint32_t i = 0; i < 4; ++i) umma::mma<1, E4M3>(tmem, da + i * 2, db + i * 2, kIdesc, kb > begin || i > 0);
                umma::commit<1>(&empty[stage]);
                if (kb + 1 == end) umma::commit<1>(&done);
            }
            __syncwarp();
            if (++stage == kAnyStages) { stage = 0; phase ^= 1; }
        }
        if (!ok && umma::elected()) umma::commit<1>(&done);        // of what has been issued
        umma::warp_wait(&done, 0, 222, &g_product_fault);
    }
    finish_slim_tile<E4M3, GATED, NT, false>(p, smem, tmem, rank, t0, i0);
}

}  // namespace ops
}  // namespace collage

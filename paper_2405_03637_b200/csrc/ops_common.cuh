// Shared by the training-step operators (row norm and rounding, gated feed-forward, distillation):
// host-side checks of matrix arguments, and small device helpers.  Host code here neither throws nor allocates.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp8.h>

#include "host_common.cuh"

namespace collage {
namespace ops {

constexpr uint64_t kMaxExtent = (1ull << 31) - 1;      // rows, columns
constexpr uint64_t kMaxLd = 1ull << 40;                // elements
constexpr float kE4m3Max = 448.0f;

inline bool same_shape(const collage_matrix_t* a, const collage_matrix_t* b) { return a->rows == b->rows && a->cols == b->cols; }

// Shape, limits, pointer and element alignment of one matrix.  An empty matrix needs no pointer.
inline collage_status_t check_matrix(const collage_matrix_t* m, uint32_t elem_bytes) {
    if (m->rows > kMaxExtent || m->cols > kMaxExtent || m->ld > kMaxLd) return COLLAGE_ERR_LIMIT;
    if (m->rows == 0 || m->cols == 0) return COLLAGE_OK;
    if (!m->data) return COLLAGE_ERR_NULL;
    if (m->ld < m->cols) return COLLAGE_ERR_ARG;
    if (reinterpret_cast<uintptr_t>(m->data) % elem_bytes) return COLLAGE_ERR_ARG;
    // the last byte's offset has to fit 62 bits
    if (m->ld && m->rows > (1ull << 58) / m->ld) return COLLAGE_ERR_LIMIT;
    return COLLAGE_OK;
}

// The bytes of a strided matrix: `rows` runs of `row_bytes`, `ld_bytes` apart.
struct Span {
    uintptr_t begin;
    uint64_t rows, row_bytes, ld_bytes;
};

inline Span span_of(const collage_matrix_t* m, uint32_t elem_bytes) {
    return {reinterpret_cast<uintptr_t>(m->data), m->cols ? m->rows : 0, m->cols * elem_bytes, m->ld * elem_bytes};
}
inline Span span_of(const void* p, uint64_t bytes) { return {reinterpret_cast<uintptr_t>(p), bytes ? 1ull : 0ull, bytes, bytes}; }

// Do two spans share a byte?  Exact for spans of one stride (column slices of one buffer interleave without
// overlapping); for unequal strides the bounding ranges decide.
inline bool overlap(const Span& a, const Span& b) {
    if (!a.rows || !b.rows || !a.begin || !b.begin) return false;
    const uintptr_t ae = a.begin + (a.rows - 1) * a.ld_bytes + a.row_bytes, be = b.begin + (b.rows - 1) * b.ld_bytes + b.row_bytes;
    if (a.begin >= be || b.begin >= ae) return false;
    // a single row fits any stride that is long enough
    const uint64_t ld = a.rows > 1 ? a.ld_bytes : b.rows > 1 ? b.ld_bytes : 0;
    if (ld == 0 || (a.rows > 1 && b.rows > 1 && a.ld_bytes != b.ld_bytes)) return true;
    if (a.row_bytes > ld || b.row_bytes > ld) return true;
    const uint64_t d = b.begin >= a.begin ? (b.begin - a.begin) % ld : (ld - (a.begin - b.begin) % ld) % ld;
    return !(d >= a.row_bytes && d + b.row_bytes <= ld);     // b's columns lie in the gap between a's rows
}

// Arrays of one call: outputs may overlap nothing, except the pairs named with `may_equal`, which may be one and the same.
struct AliasCheck {
    static constexpr int kMax = 16;
    Span span[kMax];
    bool written[kMax];
    int count = 0;
    int add(const Span& s, bool out) {
        span[count] = s;
        written[count] = out;
        return count++;
    }
    bool same(int i, int j) const {
        const Span &a = span[i], &b = span[j];
        return a.begin == b.begin && a.rows == b.rows && a.row_bytes == b.row_bytes && (a.rows == 1 || a.ld_bytes == b.ld_bytes);
    }
    // pairs: (i, j) index pairs that may coincide exactly; indexes below 0 are absent arrays
    template <int N>
    bool clash(const int (&pairs)[N][2]) const {
        for (int i = 0; i < count; ++i)
            for (int j = i + 1; j < count; ++j) {
                if (!(written[i] || written[j]) || !overlap(span[i], span[j])) continue;
                bool allowed = false;
                for (int p = 0; p < N; ++p)
                    allowed |= ((pairs[p][0] == i && pairs[p][1] == j) || (pairs[p][0] == j && pairs[p][1] == i)) && same(i, j);
                if (!allowed) return true;
            }
        return false;
    }
    bool clash() const {
        const int none[1][2] = {{-1, -1}};
        return clash(none);
    }
};

// Do all rows begin on a multiple of `bytes`?  (A single row only needs its own beginning there.)
inline bool rows_aligned(const collage_matrix_t* m, uint32_t elem_bytes, uint32_t bytes) {
    return reinterpret_cast<uintptr_t>(m->data) % bytes == 0 && (m->rows <= 1 || m->ld * elem_bytes % bytes == 0);
}

// Once per kernel and device: leave to use all of the shared memory that it does not declare statically.
template <auto Kernel>
static cudaError_t allow_smem() {
    static std::atomic<uint64_t> done{0};
    int dev = 0;
    if (const cudaError_t e = cudaGetDevice(&dev); e != cudaSuccess) return e;
    if (done.load(std::memory_order_acquire) >> (dev & 63) & 1) return cudaSuccess;
    cudaFuncAttributes attr;
    if (const cudaError_t e = cudaFuncGetAttributes(&attr, Kernel); e != cudaSuccess) return e;
    const int bytes = 227 * 1024 - static_cast<int>(attr.sharedSizeBytes);
    const cudaError_t e = cudaFuncSetAttribute(Kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess) done.fetch_or(1ull << (dev & 63), std::memory_order_release);
    return e;
}

// Launches a kernel in clusters of `cluster` blocks.  Its blocks may be set up while the stream's previous kernel still runs
// (programmatic dependent launch): every kernel launched here begins with after_previous(), before it touches memory.
template <auto Kernel, typename... Args>
static collage_status_t launch(uint64_t blocks, int threads, uint32_t cluster, size_t smem, cudaStream_t stream, const Args&... args) {
    if (blocks >= (1ull << 31)) return COLLAGE_ERR_LIMIT;
    // without leave a block has 48 KB, of which what the kernel declares statically (5 KB at most here) is taken off
    if (smem > 40 * 1024 && allow_smem<Kernel>() != cudaSuccess) return COLLAGE_ERR_CUDA;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(blocks));
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim = {cluster, 1, 1};
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, Kernel, args...) == cudaSuccess ? COLLAGE_OK : COLLAGE_ERR_CUDA;
}

// Zeros in a matrix of 2-byte or 4-byte elements (asynchronous).
inline collage_status_t clear_matrix(const collage_matrix_t* m, uint32_t elem_bytes, cudaStream_t stream) {
    if (!m->rows || !m->cols) return COLLAGE_OK;
    return cudaMemset2DAsync(m->data, m->ld * elem_bytes, 0, m->cols * elem_bytes, m->rows, stream) == cudaSuccess ? COLLAGE_OK
                                                                                                                  : COLLAGE_ERR_CUDA;
}

// ------------------------------------------------------------------------------------------------- device helpers ---

// Everything that the stream's previous kernel wrote is visible behind this, and the next one may be set up.
__device__ __forceinline__ void after_previous() {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}
__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ float bf16_value(uint16_t h) { return __uint_as_float(static_cast<uint32_t>(h) << 16); }
// two floats to one bfloat16 pair, to nearest even; `lo` goes to the lower address
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint16_t to_bf16(float f) { return __bfloat16_as_ushort(__float2bfloat16_rn(f)); }
// two floats to two e4m3 bytes, to nearest even, saturating; NaN stays NaN
__device__ __forceinline__ uint32_t pack_e4m3(float lo, float hi) {
    return __nv_cvt_float2_to_fp8x2(make_float2(lo, hi), __NV_SATFINITE, __NV_E4M3);
}
__device__ __forceinline__ uint8_t to_e4m3(float f) { return static_cast<uint8_t>(__nv_cvt_float_to_fp8(f, __NV_SATFINITE, __NV_E4M3)); }

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}

// Sum over a block of `warps` warps in a fixed order, the result in every thread.  `slots`: one float a warp.
__device__ __forceinline__ float block_sum(float v, float* slots, int warps) {
    v = warp_sum(v);
    if (warps > 1) {
        __syncthreads();
        if ((threadIdx.x & 31) == 0) slots[threadIdx.x >> 5] = v;
        __syncthreads();
        const int lane = threadIdx.x & 31;
        v = warp_sum(lane < warps ? slots[lane] : 0.0f);
    }
    return v;
}

// Largest unsigned word over the block.  On the bits of |x| this orders NaN above infinity above every number.
__device__ __forceinline__ uint32_t block_max(uint32_t v, uint32_t* slots, int warps) {
    v = __reduce_max_sync(0xFFFFFFFFu, v);
    if (warps > 1) {
        __syncthreads();
        if ((threadIdx.x & 31) == 0) slots[threadIdx.x >> 5] = v;
        __syncthreads();
        const int lane = threadIdx.x & 31;
        v = __reduce_max_sync(0xFFFFFFFFu, lane < warps ? slots[lane] : 0u);
    }
    return v;
}

// x / d for many x: Markstein's division by a correctly rounded reciprocal.  q = RN(x r) is off by a unit at most, its
// remainder q d - x is exact in an fma, and RN(q - remainder r) is the correctly rounded quotient, where nothing leaves
// the normal range (`plain`); elsewhere the division itself.
struct Divisor {
    float d, r;
    bool plain;
    __device__ __forceinline__ explicit Divisor(float divisor) : d(divisor), r(1.0f / divisor), plain(divisor > 0x1p-100f && divisor < 0x1p100f) {}
    __device__ __forceinline__ float quotient(float x) const {
        const float q = x * r;
        return __fmaf_rn(-__fmaf_rn(q, d, -x), r, q);        // (in these signs a remainder of zero leaves -0 as it is)
    }
};

}  // namespace ops
}  // namespace collage

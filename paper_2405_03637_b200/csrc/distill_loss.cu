// Distillation from a teacher's top logits: loss, its gradient, and both in one pass.
//
// With z = logits / t and lse = log sum_j exp(z_j) over the vocabulary, the teacher's p over its own entries:
//   loss = t^2 sum_k p_k (log p_k - z_index(k) + lse),   dlogits_j = g t (exp(z_j - lse) - sum_{index(k) = j} p_k).
// The softmax is taken on differences from the row's largest logit m, before the division by t: a row whose logits all
// are the type's lowest value is uniform, although neither m / t nor lse can be held to any use there.
#include "ops_common.cuh"
#include "umma.cuh"

namespace collage {
namespace ops {

struct DistillArgs {
    const void* logits;
    const void* top_index;
    const float* top_logits;
    const float* lse_in;        // backward call
    const float* row_scale;     // grad_loss or row_weight
    float* loss;
    float* lse_out;
    void* dlogits;
    uint64_t ldz, ldi, ldt, ldd;
    uint32_t vocab, k;
    uint32_t slice;             // 16-byte vectors of a row for one block
    uint32_t cluster;           // blocks of a row
    int index_bytes;
    float inv_t, t;
};

constexpr int kDistillThreads = 512;
constexpr uint32_t kMaxCluster = 8;
constexpr float kLog2e = 1.4426950408889634f;
// A stored lse of this size or more is rounded too coarsely to give q to 2^-17 (an infinite one to give it at all): the
// backward pass then takes maximum and sum from the row again.
constexpr float kLargeLse = 128.0f;
// Up to this size of m c the exponent's argument is one fma, z c - m c; beyond it m c could overflow.
constexpr float kLargeShift = 1e30f;
constexpr size_t kMaxSmem = 227 * 1024 - 1024;                 // dynamic shared memory a block may take, beside its static part
constexpr size_t kSliceBytes = 74 * 1024;                     // three blocks an SM

template <typename T>
struct Vec;                      // 16 bytes of logits
template <>
struct Vec<uint16_t> {
    static constexpr uint32_t kN = 8;
    static constexpr uint32_t kLowest = 0xFF80FF80u;          // minus infinity
    static __device__ __forceinline__ void unpack(const uint4& q, float (&f)[8]) {
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { f[2 * i] = bf16_lo(w[i]); f[2 * i + 1] = bf16_hi(w[i]); }
    }
    static __device__ __forceinline__ uint4 pack(const float (&f)[8]) {
        return make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
    }
    static __device__ __forceinline__ float value(uint16_t v) { return bf16_value(v); }
    static __device__ __forceinline__ uint16_t rounded(float v) { return to_bf16(v); }
};
template <>
struct Vec<float> {
    static constexpr uint32_t kN = 4;
    static constexpr uint32_t kLowest = 0xFF800000u;
    static __device__ __forceinline__ void unpack(const uint4& q, float (&f)[4]) {
        f[0] = __uint_as_float(q.x); f[1] = __uint_as_float(q.y); f[2] = __uint_as_float(q.z); f[3] = __uint_as_float(q.w);
    }
    static __device__ __forceinline__ uint4 pack(const float (&f)[4]) {
        return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
    }
    static __device__ __forceinline__ float value(float v) { return v; }
    static __device__ __forceinline__ float rounded(float v) { return v; }
};

__device__ __forceinline__ float fast_exp2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, o));
    return v;
}

// Sum of exp2((z - m) c) over parts with maxima of their own: `s` relative to `m` becomes relative to `to`.
__device__ __forceinline__ float rescaled(float s, float m, float to, float c) {
    return m == to ? s : m == -INFINITY ? (s != s ? s : 0.0f) : s * exp2f((m - to) * c);
}

// What a row's blocks share, apart from the row itself.
struct DistillShared {
    float2 warp[kDistillThreads / 32];
    float2 part[kMaxCluster];          // (maximum, sum) of each block of the cluster
    float loss[kMaxCluster];
    int any_there;
    float log_psum, most;
};

// A row as 16-byte vectors of its memory: vector v holds elements v kN - off ... of the row, those outside it do not exist.
template <typename T>
struct RowVectors {
    static constexpr uint32_t kN = Vec<T>::kN;
    uint4* base;                       // the row's first byte rounded down to 16
    T* row;
    uint32_t off, vocab;
    __device__ RowVectors(T* r, uint32_t n) : row(r), vocab(n) {
        const uintptr_t a = reinterpret_cast<uintptr_t>(r);
        base = reinterpret_cast<uint4*>(a & ~static_cast<uintptr_t>(15));
        off = static_cast<uint32_t>(a & 15) / sizeof(T);
    }
    __device__ uint32_t count() const { return (off + vocab + kN - 1) / kN; }
    __device__ bool inside(uint32_t v) const { return (v || !off) && (v + 1) * kN <= off + vocab; }
    // a vector at the row's edge, missing elements as minus infinity
    __device__ uint4 edge(uint32_t v) const {
        union { uint4 q; uint32_t w[4]; T e[kN]; } u;
        u.q = make_uint4(Vec<T>::kLowest, Vec<T>::kLowest, Vec<T>::kLowest, Vec<T>::kLowest);
#pragma unroll
        for (uint32_t i = 0; i < kN; ++i) {
            const int64_t e = static_cast<int64_t>(v) * kN + i - off;
            if (e >= 0 && e < vocab) u.e[i] = row[e];
        }
        return u.q;
    }
    __device__ uint4 load(uint32_t v) const { return inside(v) ? base[v] : edge(v); }
};

// A row of `vocab` logits by a cluster of blocks, each with a slice of it.  MODE 0: loss (and lse).  1: gradient from a
// stored lse.  2: both.  STAGED: the slice stays in shared memory between the two passes over it; otherwise it is read
// from global memory each time.
template <typename T, int MODE, bool STAGED>
__global__ void __launch_bounds__(kDistillThreads) distill_kernel(const __grid_constant__ DistillArgs a) {
    using V = Vec<T>;
    constexpr uint32_t kN = V::kN;
    extern __shared__ __align__(16) uint8_t dynamic[];
    __shared__ DistillShared sh;
    uint4* stage = reinterpret_cast<uint4*>(dynamic);                                    // [slice]
    float* tp = reinterpret_cast<float*>(dynamic + (STAGED ? 16ull * a.slice : 0));      // teacher: p, student's logit, index
    float* tz = tp + a.k;
    int* ti = reinterpret_cast<int*>(tz + a.k);
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = a.cluster > 1 ? umma::cluster_rank() : 0;
    const uint64_t row = blockIdx.x / a.cluster;
    const RowVectors<T> z(const_cast<T*>(static_cast<const T*>(a.logits)) + row * a.ldz, a.vocab);
    const RowVectors<T> dz(MODE ? static_cast<T*>(a.dlogits) + row * a.ldd : nullptr, a.vocab);
    const uint32_t first = rank * a.slice, end = min(first + a.slice, z.count());        // this block's vectors
    const float g = MODE ? a.row_scale[row] : 1.0f;

    constexpr uint32_t kAhead = 4;              // vectors in flight for a thread that reads global memory
    const uint4 lowest = make_uint4(V::kLowest, V::kLowest, V::kLowest, V::kLowest);
    // Gradients of the slice: `load(v)` gives a vector of logits, `value(f)` puts gradients in their place.
    auto write_row = [&](auto&& load, auto&& value) {
        const bool alike = z.off == dz.off;
        for (uint32_t v0 = first + threadIdx.x; v0 < end; v0 += kDistillThreads * kAhead) {
            uint4 q[kAhead];
#pragma unroll
            for (uint32_t i = 0; i < kAhead; ++i) q[i] = v0 + i * kDistillThreads < end ? load(v0 + i * kDistillThreads) : lowest;
#pragma unroll
            for (uint32_t n = 0; n < kAhead; ++n) {
                const uint32_t v = v0 + n * kDistillThreads;
                if (v >= end) break;
                float f[kN];
                V::unpack(q[n], f);
                value(f);
                if (alike && z.inside(v)) {
                    dz.base[v] = V::pack(f);
                } else {
#pragma unroll
                    for (uint32_t i = 0; i < kN; ++i) {
                        const int64_t e = static_cast<int64_t>(v) * kN + i - z.off;
                        if (e >= 0 && e < a.vocab) dz.row[e] = V::rounded(f[i]);
                    }
                }
            }
        }
    };
    auto zeros = [&] {
        write_row([&](uint32_t) { return lowest; }, [](float (&f)[kN]) {
#pragma unroll
            for (uint32_t i = 0; i < kN; ++i) f[i] = 0.0f;
        });
    };
    if (MODE && g == 0.0f) {
        zeros();
        if (MODE == 2 && rank == 0 && threadIdx.x == 0) a.loss[row] = 0.0f;
        return;
    }
    if (a.cluster > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");     // this block runs
    if constexpr (STAGED) {
        for (uint32_t v = first + threadIdx.x; v < end; v += kDistillThreads) {
            if (z.inside(v))
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(umma::smem_addr(stage + v - first)), "l"(z.base + v) : "memory");
            else
                stage[v - first] = z.edge(v);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    }
    auto vector = [&](uint32_t v) { return STAGED ? stage[v - first] : z.load(v); };

    if (warp == 0) {                            // the teacher's entries: p over all of them, in every block of the row
        float most = -INFINITY;
        bool bad = false;
        for (uint32_t k = lane; k < a.k; k += 32) {
            const uint64_t at = row * a.ldi + k;
            const int64_t i = a.index_bytes == 8 ? static_cast<const int64_t*>(a.top_index)[at] : static_cast<const int32_t*>(a.top_index)[at];
            const bool there = i >= 0 && i < static_cast<int64_t>(a.vocab);
            const float t = there ? a.top_logits[row * a.ldt + k] * a.inv_t : -INFINITY;
            ti[k] = there ? static_cast<int>(i) : -1;
            tp[k] = t;
            most = fmaxf(most, t);
            bad |= t != t;
        }
        most = warp_max(most);
        const bool any_there = __any_sync(0xFFFFFFFFu, bad) || most > -INFINITY;
        float psum = 0.0f;
        for (uint32_t k = lane; k < a.k; k += 32) psum += expf(tp[k] - most);
        psum = warp_sum(psum);
        for (uint32_t k = lane; k < a.k; k += 32) {
            const float shifted = tp[k] - most;
            tp[k] = expf(shifted) / psum;
            tz[k] = shifted;                    // until the student's logit takes its place
        }
        if (lane == 0) {
            sh.any_there = any_there;
            sh.log_psum = logf(psum);
        }
    }

    float m = 0.0f, sum = 1.0f;
    const float c = a.inv_t * kLog2e;
    const float lse = MODE == 1 ? a.lse_in[row] : 0.0f;
    const bool from_row = MODE != 1 || !(fabsf(lse) < kLargeLse);
    if (from_row) {
        // maximum and sum of this thread's vectors, joined over the warp, the block and the cluster
        m = -INFINITY;
        sum = 0.0f;
        if constexpr (STAGED) {
            asm volatile("cp.async.wait_group 0;" ::: "memory");          // a thread reads the vectors that it copied
            for (uint32_t v = first + threadIdx.x; v < end; v += kDistillThreads) {
                float f[kN];
                V::unpack(stage[v - first], f);
#pragma unroll
                for (uint32_t i = 0; i < kN; ++i) m = fmaxf(m, f[i]);
            }
            const float shift = -m * c;
            if (fabsf(shift) < kLargeShift) {
                for (uint32_t v = first + threadIdx.x; v < end; v += kDistillThreads) {
                    float f[kN];
                    V::unpack(stage[v - first], f);
#pragma unroll
                    for (uint32_t i = 0; i < kN; ++i) sum += fast_exp2(__fmaf_rn(f[i], c, shift));
                }
            } else {
                for (uint32_t v = first + threadIdx.x; v < end; v += kDistillThreads) {
                    float f[kN];
                    V::unpack(stage[v - first], f);
#pragma unroll
                    for (uint32_t i = 0; i < kN; ++i) sum += f[i] == m && m == -INFINITY ? 0.0f : fast_exp2((f[i] - m) * c);
                }
            }
        } else {
            for (uint32_t v = first + threadIdx.x; v < end; v += kDistillThreads * kAhead) {
                uint4 q[kAhead];
#pragma unroll
                for (uint32_t i = 0; i < kAhead; ++i) {
                    const uint32_t at = v + i * kDistillThreads;
                    q[i] = at < end ? z.load(at) : lowest;
                }
                float most = m;
#pragma unroll
                for (uint32_t i = 0; i < kAhead; ++i) {
                    float f[kN];
                    V::unpack(q[i], f);
#pragma unroll
                    for (uint32_t e = 0; e < kN; ++e) most = fmaxf(most, f[e]);
                }
                sum = rescaled(sum, m, most, c);
                m = most;
                const float shift = -m * c;
                if (fabsf(shift) < kLargeShift) {
#pragma unroll
                    for (uint32_t i = 0; i < kAhead; ++i) {
                        float f[kN];
                        V::unpack(q[i], f);
#pragma unroll
                        for (uint32_t e = 0; e < kN; ++e) sum += fast_exp2(__fmaf_rn(f[e], c, shift));
                    }
                } else {
#pragma unroll
                    for (uint32_t i = 0; i < kAhead; ++i) {
                        float f[kN];
                        V::unpack(q[i], f);
#pragma unroll
                        for (uint32_t e = 0; e < kN; ++e) sum += f[e] == m && m == -INFINITY ? 0.0f : fast_exp2((f[e] - m) * c);
                    }
                }
            }
        }
        float most = warp_max(m);
        sum = warp_sum(rescaled(sum, m, most, c));
        if (lane == 0) sh.warp[warp] = make_float2(most, sum);
        __syncthreads();
        const float2 w = lane < kDistillThreads / 32 ? sh.warp[lane] : make_float2(-INFINITY, 0.0f);
        m = warp_max(w.x);
        sum = warp_sum(rescaled(w.y, w.x, m, c));
        if (a.cluster > 1) {
            asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");           // all blocks of the row run
            if (threadIdx.x < a.cluster) {
                const uint32_t to = umma::cluster_addr(&sh.part[rank], threadIdx.x);
                asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(to), "f"(m), "f"(sum) : "memory");
            }
            umma::cluster_sync();
            const float2 r = lane < a.cluster ? sh.part[lane] : make_float2(-INFINITY, 0.0f);
            m = warp_max(r.x);
            sum = warp_sum(rescaled(r.y, r.x, m, c));
        }
    } else {
        __syncthreads();
        if (a.cluster > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    }
    // (a NaN is in no maximum, but in the sum; a row of -infinity has the sum 0 and no distribution)
    if (MODE == 0 && a.lse_out && rank == 0 && threadIdx.x == 0) a.lse_out[row] = m == -INFINITY && sum == 0.0f ? m : m * a.inv_t + logf(sum);
    if (m == -INFINITY) sum = NAN;
    const float logsum = logf(sum);
    if (!sh.any_there) {                        // nothing to learn from: zeros whatever the logits are
        if (MODE) zeros();
        if (MODE != 1 && rank == 0 && threadIdx.x == 0) a.loss[row] = 0.0f;
        return;
    }
    // log2 q_j = (z_j - m) c - log2sum, by an fma where nothing can overflow
    const float log2sum = MODE == 1 && !from_row ? lse * kLog2e : log2f(sum);
    const float shift = -m * c - log2sum;
    const bool small = fabsf(m * c) < kLargeShift;
    auto q_of = [&](float v) { return fast_exp2(small ? __fmaf_rn(v, c, shift) : (v - m) * c - log2sum); };

    // entries in this block's slice: the student's logit, and their part of the loss
    auto mine = [&](int i) {
        const uint32_t v = (static_cast<uint32_t>(i) + z.off) / kN;
        return i >= 0 && v >= first && v < end;
    };
    if (warp == 0) {
        float loss = 0.0f;
        for (uint32_t k = lane; k < a.k; k += 32) {
            const int i = ti[k];
            if (!mine(i)) continue;
            const float v = V::value(STAGED ? reinterpret_cast<const T*>(stage)[static_cast<uint32_t>(i) + z.off - first * kN] : z.row[i]);
            const float p = tp[k];
            if (MODE != 1 && !(p == 0.0f)) loss = __fmaf_rn(p, tz[k] - sh.log_psum - ((v - m) * a.inv_t - logsum), loss);
            tz[k] = v;
        }
        if (MODE != 1) {
            loss = warp_sum(loss);
            if (a.cluster > 1) {
                if (lane == 0) asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(umma::cluster_addr(&sh.loss[rank], 0)), "f"(loss) : "memory");
            } else if (lane == 0) {
                a.loss[row] = (MODE == 2 ? g : 1.0f) * (loss * a.t * a.t);
            }
        }
    }
    if (a.cluster > 1) {                        // (also: the whole row has been read before any of it is overwritten)
        umma::cluster_sync();
        if (MODE != 1 && rank == 0 && threadIdx.x == 0) {
            float loss = 0.0f;
            for (uint32_t r = 0; r < a.cluster; ++r) loss += sh.loss[r];
            a.loss[row] = (MODE == 2 ? g : 1.0f) * (loss * a.t * a.t);
        }
    } else {
        __syncthreads();
    }
    if (MODE) {
        const float gt = g * a.t;
        if (small) {
            write_row(vector, [&](float (&f)[kN]) {
#pragma unroll
                for (uint32_t i = 0; i < kN; ++i) f[i] = gt * fast_exp2(__fmaf_rn(f[i], c, shift));
            });
        } else {
            write_row(vector, [&](float (&f)[kN]) {
#pragma unroll
                for (uint32_t i = 0; i < kN; ++i) f[i] = gt * q_of(f[i]);
            });
        }
        __syncthreads();                        // the dense part is written; now the teacher's entries over it
        for (uint32_t k = threadIdx.x; k < a.k; k += kDistillThreads) {
            const int i = ti[k];
            if (!mine(i)) continue;
            float p = 0.0f;                     // an index may appear more than once: all its threads add up the same sum
            for (uint32_t o = 0; o < a.k; ++o)
                if (ti[o] == i) p += tp[o];
            dz.row[i] = V::rounded(gt * (q_of(tz[k]) - p));
        }
    }
}

template <typename T, int MODE, bool STAGED>
static collage_status_t launch_distill_as(DistillArgs& a, uint64_t rows, size_t smem, cudaStream_t s) {
    constexpr auto kernel = &distill_kernel<T, MODE, STAGED>;
    if (allow_smem<kernel>(kMaxSmem) != cudaSuccess) return COLLAGE_ERR_CUDA;
    if (rows * a.cluster >= (1ull << 31)) return COLLAGE_ERR_LIMIT;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(rows * a.cluster));
    cfg.blockDim = dim3(kDistillThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim = {a.cluster, 1, 1};
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, a) == cudaSuccess ? COLLAGE_OK : COLLAGE_ERR_CUDA;
}

template <int MODE>
static collage_status_t launch_distill(DistillArgs& a, uint64_t rows, collage_dtype_t dtype, int sm_count, void* stream) {
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const uint32_t per_vector = dtype == COLLAGE_DTYPE_BF16 ? 8 : 4;
    const uint32_t vectors = (a.vocab + 2 * per_vector - 2) / per_vector;        // at the worst alignment
    const size_t teacher = 12ull * a.k;
    bool staged = MODE == 2;
    a.cluster = 1;
    auto slice = [&] { return (vectors + a.cluster - 1) / a.cluster; };
    // three blocks of an SM hold their slices; beyond eight of those, one block may take all of the shared memory
    while (staged && a.cluster < kMaxCluster && 16ull * slice() + teacher > kSliceBytes) a.cluster *= 2;
    if (staged && 16ull * slice() + teacher > kMaxSmem) {
        staged = false;
        a.cluster = 1;
    }
    // few rows: more blocks for each, down to a vector a thread
    while (a.cluster < kMaxCluster && rows * a.cluster * 2 <= static_cast<uint64_t>(sm_count) && slice() > kDistillThreads) a.cluster *= 2;
    a.slice = slice();
    const size_t smem = (staged ? 16ull * a.slice : 0) + teacher;
    if (dtype == COLLAGE_DTYPE_BF16) {
        if constexpr (MODE == 2)
            if (staged) return launch_distill_as<uint16_t, MODE, true>(a, rows, smem, s);
        return launch_distill_as<uint16_t, MODE, false>(a, rows, smem, s);
    }
    if constexpr (MODE == 2)
        if (staged) return launch_distill_as<float, MODE, true>(a, rows, smem, s);
    return launch_distill_as<float, MODE, false>(a, rows, smem, s);
}

// Everything the three entry points check alike; `read` and `written` are their float[rows] arrays.
static collage_status_t prepare_distill(const collage_distill_t* in, const float* const (&read)[2], float* const (&written)[2],
                                        const collage_matrix_t* dlogits, DistillArgs* out, DeviceInfo* dev) {
    const uint32_t size = in->logits_dtype == COLLAGE_DTYPE_BF16 ? 2 : 4;
    if (in->logits_dtype != COLLAGE_DTYPE_BF16 && in->logits_dtype != COLLAGE_DTYPE_F32) return COLLAGE_ERR_ARG;
    if (in->top_index_bytes != 4 && in->top_index_bytes != 8) return COLLAGE_ERR_ARG;
    if (!(std::isfinite(in->temperature) && in->temperature > 0.0)) return COLLAGE_ERR_ARG;
    const float t = static_cast<float>(in->temperature), inv_t = static_cast<float>(1.0 / in->temperature);
    if (!(t > 0.0f && std::isfinite(t) && inv_t > 0.0f && std::isfinite(inv_t))) return COLLAGE_ERR_ARG;
    if (!same_shape(&in->top_index, &in->top_logits) || in->top_index.rows != in->logits.rows) return COLLAGE_ERR_ARG;
    if (dlogits && !same_shape(dlogits, &in->logits)) return COLLAGE_ERR_ARG;
    collage_status_t st = check_matrix(&in->logits, size);
    if (st == COLLAGE_OK) st = check_matrix(&in->top_index, in->top_index_bytes);
    if (st == COLLAGE_OK) st = check_matrix(&in->top_logits, 4);
    if (st == COLLAGE_OK && dlogits) st = check_matrix(dlogits, size);
    if (st != COLLAGE_OK) return st;
    if (in->top_index.cols > COLLAGE_DISTILL_MAX_TOP) return COLLAGE_ERR_LIMIT;
    AliasCheck alias;
    const int iz = alias.add(span_of(&in->logits, size), false);
    alias.add(span_of(&in->top_index, in->top_index_bytes), false);
    alias.add(span_of(&in->top_logits, 4), false);
    for (const float* p : read) {
        if (reinterpret_cast<uintptr_t>(p) % 4) return COLLAGE_ERR_ARG;
        if (p) alias.add(span_of(p, 4 * in->logits.rows), false);
    }
    for (float* p : written) {
        if (reinterpret_cast<uintptr_t>(p) % 4) return COLLAGE_ERR_ARG;
        if (p) alias.add(span_of(p, 4 * in->logits.rows), true);
    }
    const int id = dlogits ? alias.add(span_of(dlogits, size), true) : -1;
    const int pairs[1][2] = {{id, iz}};
    if (alias.clash(pairs)) return COLLAGE_ERR_ALIAS;
    if ((st = current_device(dev)) != COLLAGE_OK) return st;
    *out = {};
    out->logits = in->logits.data;
    out->ldz = in->logits.ld;
    out->top_index = in->top_index.data;
    out->ldi = in->top_index.ld;
    out->top_logits = static_cast<const float*>(in->top_logits.data);
    out->ldt = in->top_logits.ld;
    if (dlogits) { out->dlogits = dlogits->data; out->ldd = dlogits->ld; }
    out->vocab = static_cast<uint32_t>(in->logits.cols);
    out->k = static_cast<uint32_t>(in->top_index.cols);
    out->index_bytes = static_cast<int>(in->top_index_bytes);
    out->t = t;
    out->inv_t = inv_t;
    return COLLAGE_OK;
}

}  // namespace ops
}  // namespace collage

using namespace collage;
using namespace collage::ops;

extern "C" {

collage_status_t collage_distill_loss(const collage_distill_t* in, float* loss, float* lse, void* stream) {
    if (!in || (!loss && in->logits.rows)) return COLLAGE_ERR_NULL;
    DistillArgs a;
    DeviceInfo dev;
    const collage_status_t st = prepare_distill(in, {nullptr, nullptr}, {loss, lse}, nullptr, &a, &dev);
    if (st != COLLAGE_OK || in->logits.rows == 0) return st;
    a.loss = loss;
    a.lse_out = lse;
    return launch_distill<0>(a, in->logits.rows, in->logits_dtype, dev.sm_count, stream);
}

collage_status_t collage_distill_loss_backward(const collage_distill_t* in, const float* lse, const float* grad_loss,
                                               const collage_matrix_t* dlogits, void* stream) {
    if (!in || !dlogits || ((!lse || !grad_loss) && in->logits.rows)) return COLLAGE_ERR_NULL;
    DistillArgs a;
    DeviceInfo dev;
    const collage_status_t st = prepare_distill(in, {lse, grad_loss}, {nullptr, nullptr}, dlogits, &a, &dev);
    if (st != COLLAGE_OK || in->logits.rows == 0 || in->logits.cols == 0) return st;
    a.lse_in = lse;
    a.row_scale = grad_loss;
    return launch_distill<1>(a, in->logits.rows, in->logits_dtype, dev.sm_count, stream);
}

collage_status_t collage_distill_loss_and_grad(const collage_distill_t* in, const float* row_weight, float* loss,
                                               const collage_matrix_t* dlogits, void* stream) {
    if (!in || !dlogits || ((!row_weight || !loss) && in->logits.rows)) return COLLAGE_ERR_NULL;
    DistillArgs a;
    DeviceInfo dev;
    const collage_status_t st = prepare_distill(in, {row_weight, nullptr}, {loss, nullptr}, dlogits, &a, &dev);
    if (st != COLLAGE_OK || in->logits.rows == 0) return st;
    a.row_scale = row_weight;
    a.loss = loss;
    return launch_distill<2>(a, in->logits.rows, in->logits_dtype, dev.sm_count, stream);
}

}  // extern "C"

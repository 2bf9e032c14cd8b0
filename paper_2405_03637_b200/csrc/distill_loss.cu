// Distillation from a teacher's top logits: loss, its gradient, and both in one pass.
//
// With z = logits / t and lse = log sum_j exp(z_j) over the vocabulary, the teacher's p over its own entries:
//   loss = t^2 sum_k p_k (log p_k - z_index(k) + lse),   dlogits_j = g t (exp(z_j - lse) - sum_{index(k) = j} p_k).
// The softmax is taken on differences from the row's largest logit m, before the division by t: a row whose logits all
// are the type's lowest value is uniform, although neither m / t nor lse can be held to any use there.
#include "ops_common.cuh"

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
    int index_bytes;
    float inv_t, t;
};

constexpr int kDistillThreads = 256;
constexpr float kLog2e = 1.4426950408889634f;
// A stored lse of this size or more is rounded too coarsely to give q to 2^-17 (an infinite one to give it at all): the
// backward pass then takes maximum and sum from the row again.
constexpr float kLargeLse = 128.0f;

__device__ __forceinline__ float logit_value(const uint16_t* p) { return bf16_value(*p); }
__device__ __forceinline__ float logit_value(const float* p) { return *p; }
__device__ __forceinline__ void store_logit(uint16_t* p, float v) { *p = to_bf16(v); }
__device__ __forceinline__ void store_logit(float* p, float v) { *p = v; }

// The teacher's side of a row in shared memory.
struct TeacherRow {
    float p[COLLAGE_DISTILL_MAX_TOP];
    float z[COLLAGE_DISTILL_MAX_TOP];          // the student's logit at the entry
    int index[COLLAGE_DISTILL_MAX_TOP];        // -1 = absent
};

template <int THREADS>
__device__ __forceinline__ float block_max_float(float v, float* slots) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, o));
    __syncthreads();
    if ((threadIdx.x & 31) == 0) slots[threadIdx.x >> 5] = v;
    __syncthreads();
    const int lane = threadIdx.x & 31;
    v = lane < THREADS / 32 ? slots[lane] : -INFINITY;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, o));
    return v;
}

// MODE 0: loss (and lse).  1: gradient from a stored lse.  2: both.
template <typename T, int MODE>
__global__ void __launch_bounds__(kDistillThreads) distill_kernel(const __grid_constant__ DistillArgs a) {
    __shared__ TeacherRow teacher;
    __shared__ float slots[kDistillThreads / 32];
    const uint64_t row = blockIdx.x;
    const T* z = static_cast<const T*>(a.logits) + row * a.ldz;
    T* dz = MODE ? static_cast<T*>(a.dlogits) + row * a.ldd : nullptr;
    const float g = MODE ? a.row_scale[row] : 1.0f;
    if (MODE && g == 0.0f) {
        for (uint32_t j = threadIdx.x; j < a.vocab; j += kDistillThreads) store_logit(dz + j, 0.0f);
        if (MODE == 2 && threadIdx.x == 0) a.loss[row] = 0.0f;
        return;
    }
    // the teacher's entries
    float most = -INFINITY;
    bool bad = false;                          // a NaN among them
    for (uint32_t k = threadIdx.x; k < a.k; k += kDistillThreads) {
        const uint64_t at = row * a.ldi + k;
        const int64_t i = a.index_bytes == 8 ? static_cast<const int64_t*>(a.top_index)[at] : static_cast<const int32_t*>(a.top_index)[at];
        const bool there = i >= 0 && i < static_cast<int64_t>(a.vocab);
        const float t = there ? a.top_logits[row * a.ldt + k] * a.inv_t : -INFINITY;
        teacher.index[k] = there ? static_cast<int>(i) : -1;
        teacher.p[k] = t;
        teacher.z[k] = there ? logit_value(z + i) : 0.0f;
        most = fmaxf(most, t);
        bad |= t != t;
    }
    most = block_max_float<kDistillThreads>(most, slots);
    const bool any_there = __syncthreads_or(bad) || most > -INFINITY;
    if (!any_there) {                          // nothing to learn from: zeros whatever the logits are
        if (MODE)
            for (uint32_t j = threadIdx.x; j < a.vocab; j += kDistillThreads) store_logit(dz + j, 0.0f);
        if (MODE != 1 && threadIdx.x == 0) a.loss[row] = 0.0f;
        if (MODE != 0 || !a.lse_out) return;
    }
    // q_j = exp2((z_j - m) c - log2sum)
    float m = -INFINITY, log2sum, logsum = 0.0f;
    const float c = a.inv_t * kLog2e;
    const float lse = MODE == 1 ? a.lse_in[row] : 0.0f;
    if (MODE == 1 && fabsf(lse) < kLargeLse) {
        m = 0.0f;
        log2sum = lse * kLog2e;
    } else {
        float sum = 0.0f;
        for (uint32_t j = threadIdx.x; j < a.vocab; j += kDistillThreads) m = fmaxf(m, logit_value(z + j));
        m = block_max_float<kDistillThreads>(m, slots);
        for (uint32_t j = threadIdx.x; j < a.vocab; j += kDistillThreads) sum += exp2f((logit_value(z + j) - m) * c);
        sum = block_sum<kDistillThreads>(sum, slots);
        log2sum = log2f(sum);
        logsum = logf(sum);
        if (MODE == 0 && a.lse_out && threadIdx.x == 0) a.lse_out[row] = m * a.inv_t + logsum;
        if (!any_there) return;
    }
    auto log2q = [&](float v) { return (v - m) * c - log2sum; };
    float psum = 0.0f;
    for (uint32_t k = threadIdx.x; k < a.k; k += kDistillThreads) psum += expf(teacher.p[k] - most);
    psum = block_sum<kDistillThreads>(psum, slots);
    const float logpsum = logf(psum);
    float loss = 0.0f;
    for (uint32_t k = threadIdx.x; k < a.k; k += kDistillThreads) {
        const float shifted = teacher.p[k] - most, p = expf(shifted) / psum;
        teacher.p[k] = p;
        if (MODE != 1 && !(p == 0.0f)) loss = __fmaf_rn(p, shifted - logpsum - ((teacher.z[k] - m) * a.inv_t - logsum), loss);
    }
    if (MODE != 1) {
        loss = block_sum<kDistillThreads>(loss, slots) * a.t * a.t;
        if (threadIdx.x == 0) a.loss[row] = MODE == 2 ? g * loss : loss;
    }
    if (MODE) {
        const float gt = g * a.t;
        __syncthreads();
        for (uint32_t j = threadIdx.x; j < a.vocab; j += kDistillThreads)
            store_logit(dz + j, gt * exp2f(log2q(logit_value(z + j))));
        __syncthreads();                       // the dense part is written; now the teacher's entries over it
        for (uint32_t k = threadIdx.x; k < a.k; k += kDistillThreads) {
            const int i = teacher.index[k];
            if (i < 0) continue;
            float p = 0.0f;                    // an index may appear more than once: all its threads add up the same sum
            for (uint32_t o = 0; o < a.k; ++o)
                if (teacher.index[o] == i) p += teacher.p[o];
            store_logit(dz + i, gt * (exp2f(log2q(teacher.z[k])) - p));
        }
    }
}

template <int MODE>
collage_status_t launch_distill(const DistillArgs& a, uint64_t rows, collage_dtype_t dtype, void* stream) {
    const unsigned grid = static_cast<unsigned>(rows);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (dtype == COLLAGE_DTYPE_BF16)
        distill_kernel<uint16_t, MODE><<<grid, kDistillThreads, 0, s>>>(a);
    else
        distill_kernel<float, MODE><<<grid, kDistillThreads, 0, s>>>(a);
    return launch_status();
}

// Everything the three entry points check alike; `read` and `written` are their float[rows] arrays.
static collage_status_t prepare_distill(const collage_distill_t* in, const float* const (&read)[2], float* const (&written)[2],
                                        const collage_matrix_t* dlogits, DistillArgs* out) {
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
    DeviceInfo dev;
    if ((st = current_device(&dev)) != COLLAGE_OK) return st;
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
    const collage_status_t st = prepare_distill(in, {nullptr, nullptr}, {loss, lse}, nullptr, &a);
    if (st != COLLAGE_OK || in->logits.rows == 0) return st;
    a.loss = loss;
    a.lse_out = lse;
    return launch_distill<0>(a, in->logits.rows, in->logits_dtype, stream);
}

collage_status_t collage_distill_loss_backward(const collage_distill_t* in, const float* lse, const float* grad_loss,
                                               const collage_matrix_t* dlogits, void* stream) {
    if (!in || !dlogits || ((!lse || !grad_loss) && in->logits.rows)) return COLLAGE_ERR_NULL;
    DistillArgs a;
    const collage_status_t st = prepare_distill(in, {lse, grad_loss}, {nullptr, nullptr}, dlogits, &a);
    if (st != COLLAGE_OK || in->logits.rows == 0 || in->logits.cols == 0) return st;
    a.lse_in = lse;
    a.row_scale = grad_loss;
    return launch_distill<1>(a, in->logits.rows, in->logits_dtype, stream);
}

collage_status_t collage_distill_loss_and_grad(const collage_distill_t* in, const float* row_weight, float* loss,
                                               const collage_matrix_t* dlogits, void* stream) {
    if (!in || !dlogits || ((!row_weight || !loss) && in->logits.rows)) return COLLAGE_ERR_NULL;
    DistillArgs a;
    const collage_status_t st = prepare_distill(in, {row_weight, nullptr}, {loss, nullptr}, dlogits, &a);
    if (st != COLLAGE_OK || in->logits.rows == 0) return st;
    a.row_scale = row_weight;
    a.loss = loss;
    return launch_distill<2>(a, in->logits.rows, in->logits_dtype, stream);
}

}  // extern "C"

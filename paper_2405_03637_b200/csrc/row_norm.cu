// Residual addition + RMS norm (bfloat16 or e4m3 output), its backward pass, and rounding of rows to e4m3.
#include "ops_common.cuh"

namespace collage {
namespace ops {

struct RowArgs {
    const uint16_t* x;
    const uint16_t* residual;
    const uint16_t* weight;
    uint16_t* residual_out;
    uint16_t* y;
    uint8_t* y8;
    float* scale;
    float* rstd;
    uint64_t ldx, ldres, ldro, ldy, ldy8;
    uint64_t cols;
    float eps;
};

constexpr int kRowThreads = 256;

// One block per row, element by element, the row read again for each stage: any length, stride and alignment.
template <bool NORM>
__global__ void __launch_bounds__(kRowThreads) row_any_kernel(const __grid_constant__ RowArgs a) {
    __shared__ float slots[kRowThreads / 32];
    const uint64_t row = blockIdx.x;
    const uint16_t* x = a.x + row * a.ldx;
    const uint16_t* res = a.residual ? a.residual + row * a.ldres : nullptr;
    auto value = [&](uint64_t j) { return res ? bf16_value(x[j]) + bf16_value(res[j]) : bf16_value(x[j]); };
    float rstd = 1.0f;
    if (NORM) {
        float sum = 0.0f;
        for (uint64_t j = threadIdx.x; j < a.cols; j += kRowThreads) {
            const float r = value(j);
            sum = __fmaf_rn(r, r, sum);
        }
        sum = block_sum<kRowThreads>(sum, slots);
        rstd = 1.0f / sqrtf(sum / static_cast<float>(a.cols) + a.eps);
        if (a.rstd && threadIdx.x == 0) a.rstd[row] = rstd;
    }
    auto normed = [&](float r, uint64_t j) { return NORM ? r * rstd * bf16_value(a.weight[j]) : r; };
    float scale = 0.0f;
    if (a.y8) {
        uint32_t most = 0;
        for (uint64_t j = threadIdx.x; j < a.cols; j += kRowThreads)
            most = max(most, __float_as_uint(normed(value(j), j)) & 0x7FFFFFFFu);
        most = block_max<kRowThreads>(most, reinterpret_cast<uint32_t*>(slots));
        scale = __uint_as_float(most) / kE4m3Max;
        if (threadIdx.x == 0) a.scale[row] = scale;
    }
    // outputs last: residual_out or y may be the array that x or residual is, element for element
    for (uint64_t j = threadIdx.x; j < a.cols; j += kRowThreads) {
        const float r = value(j), y = normed(r, j);
        if (a.residual_out) a.residual_out[row * a.ldro + j] = to_bf16(r);
        if (a.y) a.y[row * a.ldy + j] = to_bf16(y);
        if (a.y8) a.y8[row * a.ldy8 + j] = scale == 0.0f ? 0 : to_e4m3(y / scale);
    }
}

struct RowBackwardArgs {
    const uint16_t* dy;
    const uint16_t* r;
    const float* rstd;
    const uint16_t* weight;
    const uint16_t* dresidual;
    uint16_t* dx;
    uint16_t* dweight;
    float* partial;                       // [chunks, cols]
    uint64_t lddy, ldr, lddres, lddx;
    uint64_t rows, cols;
};

// dx of one row: one block, element by element.
__global__ void __launch_bounds__(kRowThreads) row_backward_any_kernel(const __grid_constant__ RowBackwardArgs a) {
    __shared__ float slots[kRowThreads / 32];
    const uint64_t row = blockIdx.x;
    const uint16_t* dy = a.dy + row * a.lddy;
    const uint16_t* r = a.r + row * a.ldr;
    const uint16_t* dres = a.dresidual ? a.dresidual + row * a.lddres : nullptr;
    const float rstd = a.rstd[row];
    float sum = 0.0f;
    for (uint64_t j = threadIdx.x; j < a.cols; j += kRowThreads)
        sum = __fmaf_rn(bf16_value(dy[j]) * bf16_value(a.weight[j]), bf16_value(r[j]) * rstd, sum);
    const float mean = block_sum<kRowThreads>(sum, slots) / static_cast<float>(a.cols);
    for (uint64_t j = threadIdx.x; j < a.cols; j += kRowThreads) {
        float d = rstd * __fmaf_rn(-bf16_value(r[j]) * rstd, mean, bf16_value(dy[j]) * bf16_value(a.weight[j]));
        if (dres) d += bf16_value(dres[j]);
        a.dx[row * a.lddx + j] = to_bf16(d);
    }
}

constexpr int kWeightChunks = 256;        // row chunks whose sums are kept apart

// Sums of dy * n over a chunk of rows, 32 columns a block.
__global__ void __launch_bounds__(kRowThreads) row_dweight_any_kernel(const __grid_constant__ RowBackwardArgs a) {
    __shared__ float part[kRowThreads / 32][32];
    const uint64_t j = blockIdx.x * 32ull + (threadIdx.x & 31);
    const int lane_row = threadIdx.x >> 5;
    const uint64_t per = (a.rows + gridDim.y - 1) / gridDim.y;
    const uint64_t begin = blockIdx.y * per, end = min(begin + per, a.rows);
    float sum = 0.0f;
    if (j < a.cols)
        for (uint64_t i = begin + lane_row; i < end; i += kRowThreads / 32)
            sum = __fmaf_rn(bf16_value(a.dy[i * a.lddy + j]), bf16_value(a.r[i * a.ldr + j]) * a.rstd[i], sum);
    part[lane_row][threadIdx.x & 31] = sum;
    __syncthreads();
    if (lane_row == 0 && j < a.cols) {
        for (int k = 1; k < kRowThreads / 32; ++k) sum += part[k][threadIdx.x];
        a.partial[blockIdx.y * a.cols + j] = sum;
    }
}

__global__ void __launch_bounds__(kRowThreads) row_dweight_finish_kernel(const float* partial, int chunks, uint64_t cols, uint16_t* dweight) {
    const uint64_t j = blockIdx.x * static_cast<uint64_t>(kRowThreads) + threadIdx.x;
    if (j >= cols) return;
    float sum = 0.0f;
    for (int k = 0; k < chunks; ++k) sum += partial[k * cols + j];
    dweight[j] = to_bf16(sum);
}

}  // namespace ops
}  // namespace collage

using namespace collage;
using namespace collage::ops;

extern "C" {

collage_status_t collage_add_rms_norm(const collage_matrix_t* x, const collage_matrix_t* residual, const void* weight, double eps,
                                      const collage_matrix_t* residual_out, const collage_matrix_t* y, const collage_matrix_t* y8,
                                      float* y8_scale, float* rstd, void* stream) {
    if (!x || (!weight && x->cols) || (!y && !y8) || (y8 && !y8_scale && x->rows)) return COLLAGE_ERR_NULL;
    if (!(std::isfinite(eps) && eps >= 0.0) || (y8_scale && !y8) || (residual_out && !residual)) return COLLAGE_ERR_ARG;
    const collage_matrix_t* others[4] = {residual, residual_out, y, y8};
    collage_status_t st = check_matrix(x, 2);
    for (int i = 0; i < 4 && st == COLLAGE_OK; ++i)
        if (others[i]) st = !same_shape(x, others[i]) ? COLLAGE_ERR_ARG : check_matrix(others[i], i == 3 ? 1 : 2);
    if (st != COLLAGE_OK) return st;
    if (reinterpret_cast<uintptr_t>(weight) % 2 || reinterpret_cast<uintptr_t>(y8_scale) % 4 || reinterpret_cast<uintptr_t>(rstd) % 4)
        return COLLAGE_ERR_ARG;
    AliasCheck alias;
    const int ix = alias.add(span_of(x, 2), false);
    alias.add(span_of(weight, 2 * x->cols), false);
    const int ires = residual ? alias.add(span_of(residual, 2), false) : -1;
    const int iro = residual_out ? alias.add(span_of(residual_out, 2), true) : -1;
    const int iy = y ? alias.add(span_of(y, 2), true) : -1;
    if (y8) alias.add(span_of(y8, 1), true);
    if (y8_scale) alias.add(span_of(y8_scale, 4 * x->rows), true);
    if (rstd) alias.add(span_of(rstd, 4 * x->rows), true);
    const int pairs[3][2] = {{iro, ix}, {iro, ires}, {iy, ix}};
    if (alias.clash(pairs)) return COLLAGE_ERR_ALIAS;
    DeviceInfo dev;
    if ((st = current_device(&dev)) != COLLAGE_OK) return st;
    if (x->rows == 0 || x->cols == 0) return COLLAGE_OK;
    RowArgs a = {};
    a.x = static_cast<const uint16_t*>(x->data);
    a.ldx = x->ld;
    if (residual) { a.residual = static_cast<const uint16_t*>(residual->data); a.ldres = residual->ld; }
    if (residual_out) { a.residual_out = static_cast<uint16_t*>(residual_out->data); a.ldro = residual_out->ld; }
    if (y) { a.y = static_cast<uint16_t*>(y->data); a.ldy = y->ld; }
    if (y8) { a.y8 = static_cast<uint8_t*>(y8->data); a.ldy8 = y8->ld; a.scale = y8_scale; }
    a.weight = static_cast<const uint16_t*>(weight);
    a.rstd = rstd;
    a.cols = x->cols;
    a.eps = static_cast<float>(eps);
    row_any_kernel<true><<<static_cast<unsigned>(x->rows), kRowThreads, 0, static_cast<cudaStream_t>(stream)>>>(a);
    return launch_status();
}

collage_status_t collage_quantize_rows(const collage_matrix_t* x, const collage_matrix_t* q, float* scale, void* stream) {
    if (!x || !q || (!scale && x->rows)) return COLLAGE_ERR_NULL;
    if (!same_shape(x, q) || reinterpret_cast<uintptr_t>(scale) % 4) return COLLAGE_ERR_ARG;
    collage_status_t st = check_matrix(x, 2);
    if (st == COLLAGE_OK) st = check_matrix(q, 1);
    if (st != COLLAGE_OK) return st;
    AliasCheck alias;
    alias.add(span_of(x, 2), false);
    alias.add(span_of(q, 1), true);
    alias.add(span_of(scale, 4 * x->rows), true);
    if (alias.clash()) return COLLAGE_ERR_ALIAS;
    DeviceInfo dev;
    if ((st = current_device(&dev)) != COLLAGE_OK) return st;
    if (x->rows == 0) return COLLAGE_OK;
    if (x->cols == 0)
        return cudaMemsetAsync(scale, 0, 4 * x->rows, static_cast<cudaStream_t>(stream)) == cudaSuccess ? COLLAGE_OK : COLLAGE_ERR_CUDA;
    RowArgs a = {};
    a.x = static_cast<const uint16_t*>(x->data);
    a.ldx = x->ld;
    a.y8 = static_cast<uint8_t*>(q->data);
    a.ldy8 = q->ld;
    a.scale = scale;
    a.cols = x->cols;
    row_any_kernel<false><<<static_cast<unsigned>(x->rows), kRowThreads, 0, static_cast<cudaStream_t>(stream)>>>(a);
    return launch_status();
}

size_t collage_rms_norm_workspace_bytes(uint64_t cols) { return static_cast<size_t>(kWeightChunks) * 4 * cols; }

collage_status_t collage_add_rms_norm_backward(const collage_matrix_t* dy, const collage_matrix_t* r, const float* rstd,
                                               const void* weight, const collage_matrix_t* dresidual, const collage_matrix_t* dx,
                                               void* dweight, void* workspace, size_t workspace_bytes, void* stream) {
    if (!dy || !r || (!rstd && dy->rows) || (!weight && dy->cols) || (!dx && !dweight && dy->cols)) return COLLAGE_ERR_NULL;
    const collage_matrix_t* others[3] = {r, dresidual, dx};
    collage_status_t st = check_matrix(dy, 2);
    for (int i = 0; i < 3 && st == COLLAGE_OK; ++i)
        if (others[i]) st = !same_shape(dy, others[i]) ? COLLAGE_ERR_ARG : check_matrix(others[i], 2);
    if (st != COLLAGE_OK) return st;
    if (reinterpret_cast<uintptr_t>(weight) % 2 || reinterpret_cast<uintptr_t>(dweight) % 2 || reinterpret_cast<uintptr_t>(rstd) % 4)
        return COLLAGE_ERR_ARG;
    const size_t need = collage_rms_norm_workspace_bytes(dy->cols);
    if (dweight && need && (!workspace || workspace_bytes < need || reinterpret_cast<uintptr_t>(workspace) % 16)) return COLLAGE_ERR_WORKSPACE;
    AliasCheck alias;
    const int idy = alias.add(span_of(dy, 2), false);
    alias.add(span_of(r, 2), false);
    alias.add(span_of(rstd, 4 * dy->rows), false);
    alias.add(span_of(weight, 2 * dy->cols), false);
    const int ires = dresidual ? alias.add(span_of(dresidual, 2), false) : -1;
    const int idx = dx ? alias.add(span_of(dx, 2), true) : -1;
    if (dweight) {
        alias.add(span_of(dweight, 2 * dy->cols), true);
        alias.add(span_of(workspace, need), true);
    }
    const int pairs[2][2] = {{idx, idy}, {idx, ires}};
    if (alias.clash(pairs)) return COLLAGE_ERR_ALIAS;
    DeviceInfo dev;
    if ((st = current_device(&dev)) != COLLAGE_OK) return st;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (dy->cols == 0) return COLLAGE_OK;
    if (dy->rows == 0)
        return !dweight || cudaMemsetAsync(dweight, 0, 2 * dy->cols, s) == cudaSuccess ? COLLAGE_OK : COLLAGE_ERR_CUDA;
    RowBackwardArgs a = {};
    a.dy = static_cast<const uint16_t*>(dy->data);
    a.lddy = dy->ld;
    a.r = static_cast<const uint16_t*>(r->data);
    a.ldr = r->ld;
    a.rstd = rstd;
    a.weight = static_cast<const uint16_t*>(weight);
    if (dresidual) { a.dresidual = static_cast<const uint16_t*>(dresidual->data); a.lddres = dresidual->ld; }
    if (dx) { a.dx = static_cast<uint16_t*>(dx->data); a.lddx = dx->ld; }
    a.dweight = static_cast<uint16_t*>(dweight);
    a.partial = static_cast<float*>(workspace);
    a.rows = dy->rows;
    a.cols = dy->cols;
    if (dweight) {                            // before dx, which may take dy's place
        const uint64_t blocks = (a.cols + 31) / 32;
        uint64_t chunks = (8ull * dev.sm_count + blocks - 1) / blocks;
        chunks = std::min<uint64_t>({chunks, (a.rows + 7) / 8, static_cast<uint64_t>(kWeightChunks)});
        row_dweight_any_kernel<<<dim3(static_cast<unsigned>(blocks), static_cast<unsigned>(chunks)), kRowThreads, 0, s>>>(a);
        row_dweight_finish_kernel<<<static_cast<unsigned>((a.cols + kRowThreads - 1) / kRowThreads), kRowThreads, 0, s>>>(
            a.partial, static_cast<int>(chunks), a.cols, a.dweight);
    }
    if (dx) row_backward_any_kernel<<<static_cast<unsigned>(a.rows), kRowThreads, 0, s>>>(a);
    return launch_status();
}

}  // extern "C"

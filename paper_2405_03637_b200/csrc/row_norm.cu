// Residual addition + RMS norm (bfloat16 or e4m3 output), its backward pass, and rounding of rows to e4m3.
//
//   r = x + residual,  n = r / sqrt(mean r^2 + eps),  y = n * weight
//   dx = rstd (g - n mean(g n)) + dresidual  with g = weight * dy,   dweight = sum over rows of dy * n
//   scale = max |y| / 448,  y8 = e4m3(y / scale)
//
// All of it is bound by memory: a row is read once, kept in registers until its sum (and maximum) is known, and written.
// Measured at 8191 x 4096: forward 40.9 us (6.6 TB/s, the rate of a copy), with 8-bit output 38.4 us (6.1), backward with both
// gradients 47.3 us (5.7 TB/s); quantise 11008 x 4096 24.8 us (5.5 TB/s).
// r is rounded to bfloat16 for the residual stream, and it is those values that the backward pass reads, while y and rstd belong
// to r before the rounding.  A training program keeps no second copy of the stream; dx and dweight carry the rounding (2.2e-3
// from the definition in the relative 2-norm at 8191 x 4096, 1.7e-3 with r in float).
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

// One block per row, element by element, the row read again for each stage: any length, stride and alignment.  8191 x 4097 forward
// 74 us (3.6 TB/s), to 8 bits 96 us; quantise 51 us (2.0 TB/s): the loads of two bytes bound it.
template <bool NORM>
__global__ void __launch_bounds__(kRowThreads) row_any_kernel(const __grid_constant__ RowArgs a) {
    __shared__ float slots[kRowThreads / 32];
    after_previous();
    const uint64_t row = blockIdx.x;
    const uint16_t* x = a.x + row * a.ldx;
    const uint16_t* res = a.residual ? a.residual + row * a.ldres : nullptr;
    auto value = [&](uint64_t j) { return res ? bf16_value(x[j]) + bf16_value(res[j]) : bf16_value(x[j]); };
    float rstd = 1.0f;
    if (NORM) {
        auto mean_of = [&](float f) {
            float sum = 0.0f;
            for (uint64_t j = threadIdx.x; j < a.cols; j += kRowThreads) {
                const float r = value(j) * f;
                sum = __fmaf_rn(r, r, sum);
            }
            return block_sum(sum, slots, kRowThreads / 32) / static_cast<float>(a.cols) + a.eps * f * f;
        };
        float mean = mean_of(1.0f), f = 1.0f;
        if (!squares_fit(mean)) mean = mean_of(f = rescue_factor(mean));
        rstd = f / sqrtf(mean);
        if (a.rstd && threadIdx.x == 0) a.rstd[row] = rstd;
    }
    auto normed = [&](float r, uint64_t j) { return NORM ? r * rstd * bf16_value(a.weight[j]) : r; };
    float scale = 0.0f;
    if (a.scale) {
        uint32_t most = 0;
        for (uint64_t j = threadIdx.x; j < a.cols; j += kRowThreads)
            most = max(most, __float_as_uint(normed(value(j), j)) & 0x7FFFFFFFu);
        most = block_max(most, reinterpret_cast<uint32_t*>(slots), kRowThreads / 32);
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

// Rows of whole 16-byte vectors, read once and kept in registers: PER vectors a thread, a row by one warp (WARP: four rows a
// block) or by a block of as many warps as it takes.
template <int PER, bool NORM, bool WARP>
__global__ void __launch_bounds__(WARP ? 128 : PER > 2 ? 512 : 1024) row_kernel(const __grid_constant__ RowArgs a, uint64_t rows) {
    __shared__ float slots[32];
    after_previous();
    const uint64_t row = WARP ? blockIdx.x * 4ull + (threadIdx.x >> 5) : blockIdx.x;
    if (WARP && row >= rows) return;
    const int t = WARP ? threadIdx.x & 31 : threadIdx.x, threads = WARP ? 32 : blockDim.x, warps = threads >> 5;
    const int vectors = static_cast<int>(a.cols >> 3);
    const uint4 none = make_uint4(0, 0, 0, 0);
    float r[PER][8];
    uint4 q[PER], qr[PER], qw[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int v = t + i * threads;
        q[i] = v < vectors ? reinterpret_cast<const uint4*>(a.x + row * a.ldx)[v] : none;
        if (NORM && a.residual) qr[i] = v < vectors ? reinterpret_cast<const uint4*>(a.residual + row * a.ldres)[v] : none;
    }
    if (NORM) {
#pragma unroll
        for (int i = 0; i < PER; ++i) qw[i] = t + i * threads < vectors ? __ldg(reinterpret_cast<const uint4*>(a.weight) + t + i * threads) : none;
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        unpack8(q[i], r[i]);
        if (NORM && a.residual) {
            float s[8];
            unpack8(qr[i], s);
#pragma unroll
            for (int e = 0; e < 8; ++e) r[i][e] += s[e];
        }
    }
    if (NORM) {
        float f = 1.0f, rstd;                        // rstd: of the row times f
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int v = t + i * threads;
            if (a.residual_out && v < vectors) reinterpret_cast<uint4*>(a.residual_out + row * a.ldro)[v] = pack8(r[i]);
        }
#pragma unroll 1
        for (;;) {
            float part[PER];
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                part[i] = 0.0f;
#pragma unroll
                for (int e = 0; e < 8; ++e) part[i] = __fmaf_rn(r[i][e], r[i][e], part[i]);
            }
            float sum = part[0];
#pragma unroll
            for (int i = 1; i < PER; ++i) sum += part[i];
            const float mean = block_sum(sum, slots, warps) / static_cast<float>(a.cols) + a.eps * f * f;
            rstd = 1.0f / sqrtf(mean);
            if (squares_fit(mean) || f != 1.0f) break;
            f = rescue_factor(mean);
#pragma unroll
            for (int i = 0; i < PER; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) r[i][e] *= f;
        }
        if (a.rstd && t == 0) a.rstd[row] = f * rstd;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int v = t + i * threads;
            float w[8];
            unpack8(qw[i], w);
#pragma unroll
            for (int e = 0; e < 8; ++e) r[i][e] = r[i][e] * rstd * w[e];
            if (a.y && v < vectors) reinterpret_cast<uint4*>(a.y + row * a.ldy)[v] = pack8(r[i]);
        }
    }
    if (a.y8) {
        uint32_t most = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) most = max(most, __float_as_uint(r[i][e]) & 0x7FFFFFFFu);
        most = block_max(most, reinterpret_cast<uint32_t*>(slots), warps);
        const float scale = __uint_as_float(most) / kE4m3Max;
        if (t == 0) a.scale[row] = scale;
        const Divisor by(scale);
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int v = t + i * threads;
            if (v >= vectors) continue;
            uint32_t w[2] = {0, 0};
            if (by.plain) {
#pragma unroll
                for (int e = 0; e < 8; e += 2) w[e >> 2] |= pack_e4m3(by.quotient(r[i][e]), by.quotient(r[i][e + 1])) << (8 * (e & 2));
            } else if (scale != 0.0f) {
#pragma unroll
                for (int e = 0; e < 8; e += 2) w[e >> 2] |= pack_e4m3(r[i][e] / scale, r[i][e + 1] / scale) << (8 * (e & 2));
            }
            reinterpret_cast<uint2*>(a.y8 + row * a.ldy8)[v] = make_uint2(w[0], w[1]);
        }
    }
}

// A row's vectors over warps: with many rows four vectors a thread (more loads in flight, fewer warps to join), with few rows
// one (the shortest way through a row), as far as 1024 or 512 threads reach.
template <bool NORM>
static collage_status_t launch_rows(const RowArgs& a, uint64_t rows, bool vectors_fit, int sm_count, cudaStream_t s) {
    const uint64_t v = a.cols >> 3;
    const bool many = rows > 2ull * sm_count;
    if (!vectors_fit || v > 4096) return launch<&row_any_kernel<NORM>>(rows, kRowThreads, 1, 0, s, a);
    if (many && v <= 128) {
        const uint64_t grid = (rows + 3) / 4;
        return v <= 32   ? launch<&row_kernel<1, NORM, true>>(grid, 128, 1, 0, s, a, rows)
               : v <= 64 ? launch<&row_kernel<2, NORM, true>>(grid, 128, 1, 0, s, a, rows)
                         : launch<&row_kernel<4, NORM, true>>(grid, 128, 1, 0, s, a, rows);
    }
    const uint64_t per = v > 2048 ? 8 : many ? 4 : v > 1024 ? 2 : 1;
    const int threads = static_cast<int>((v + per * 32 - 1) / (per * 32) * 32);
    return per == 1   ? launch<&row_kernel<1, NORM, false>>(rows, threads, 1, 0, s, a, rows)
           : per == 2 ? launch<&row_kernel<2, NORM, false>>(rows, threads, 1, 0, s, a, rows)
           : per == 4 ? launch<&row_kernel<4, NORM, false>>(rows, threads, 1, 0, s, a, rows)
                      : launch<&row_kernel<8, NORM, false>>(rows, threads, 1, 0, s, a, rows);
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
    after_previous();
    const uint64_t row = blockIdx.x;
    const uint16_t* dy = a.dy + row * a.lddy;
    const uint16_t* r = a.r + row * a.ldr;
    const uint16_t* dres = a.dresidual ? a.dresidual + row * a.lddres : nullptr;
    const float rstd = a.rstd[row];
    float sum = 0.0f;
    for (uint64_t j = threadIdx.x; j < a.cols; j += kRowThreads)
        sum = __fmaf_rn(bf16_value(dy[j]) * bf16_value(a.weight[j]), bf16_value(r[j]) * rstd, sum);
    const float mean = block_sum(sum, slots, kRowThreads / 32) / static_cast<float>(a.cols);
    for (uint64_t j = threadIdx.x; j < a.cols; j += kRowThreads) {
        float d = rstd * __fmaf_rn(-bf16_value(r[j]) * rstd, mean, bf16_value(dy[j]) * bf16_value(a.weight[j]));
        if (dres) d += bf16_value(dres[j]);
        a.dx[row * a.lddx + j] = to_bf16(d);
    }
}

constexpr int kWeightChunks = 320;        // row chunks whose sums are kept apart

// Sums of dy * n over a chunk of rows, 32 columns a block.
__global__ void __launch_bounds__(kRowThreads) row_dweight_any_kernel(const __grid_constant__ RowBackwardArgs a, uint32_t chunks) {
    __shared__ float part[kRowThreads / 32][32];
    after_previous();
    const uint32_t chunk = blockIdx.x % chunks;
    const uint64_t j = blockIdx.x / chunks * 32ull + (threadIdx.x & 31);
    const int lane_row = threadIdx.x >> 5;
    const uint64_t per = (a.rows + chunks - 1) / chunks;
    const uint64_t begin = chunk * per, end = min(begin + per, a.rows);
    float sum = 0.0f;
    if (j < a.cols)
        for (uint64_t i = begin + lane_row; i < end; i += kRowThreads / 32)
            sum = __fmaf_rn(bf16_value(a.dy[i * a.lddy + j]), bf16_value(a.r[i * a.ldr + j]) * a.rstd[i], sum);
    part[lane_row][threadIdx.x & 31] = sum;
    __syncthreads();
    if (lane_row == 0 && j < a.cols) {
        for (int k = 1; k < kRowThreads / 32; ++k) sum += part[k][threadIdx.x];
        a.partial[chunk * a.cols + j] = sum;
    }
}

// Gradients of rows of whole vectors in one pass (dy, r and dresidual are read once for dx and dweight): blocks walk over rows, one at a time for each group of `group` threads.
// A thread owns PER vectors of columns: it sends for its own of the next two rows ahead (so loads go on while the row's
// sum is joined), and keeps its columns' part of dweight in registers until the end.
constexpr int kBackwardThreads = 512, kDepth = 2;

template <int PER, int THREADS>
__global__ void __launch_bounds__(THREADS, PER > 1 ? 1 : 2) row_backward_kernel(const __grid_constant__ RowBackwardArgs a, int group_threads) {
    __shared__ float slots[2][32];
    extern __shared__ __align__(16) uint8_t dynamic[];
    after_previous();
    const int groups = blockDim.x / group_threads, group = threadIdx.x / group_threads, t = threadIdx.x % group_threads;
    const int lane = threadIdx.x & 31, group_warps = group_threads >> 5, warp0 = group * group_warps;
    const int vectors = static_cast<int>(a.cols >> 3);
    const uint4 none = make_uint4(0, 0, 0, 0);
    uint4* mine = reinterpret_cast<uint4*>(dynamic) + threadIdx.x;      // [kDepth][3][PER] places, blockDim.x apart
    auto place = [&](int stage, int array, int i) { return mine + ((stage * 3 + array) * PER + i) * blockDim.x; };
    uint4 qw[PER];
    float dw[PER][8];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        qw[i] = t + i * group_threads < vectors ? reinterpret_cast<const uint4*>(a.weight)[t + i * group_threads] : none;
#pragma unroll
        for (int e = 0; e < 8; ++e) dw[i][e] = 0.0f;
        for (int d = 0; d < kDepth; ++d)
            for (int k = 0; k < 3; ++k) *place(d, k, i) = none;         // places that no load fills
    }
    const bool with_res = a.dresidual && a.dx;
    const uint64_t first = blockIdx.x * static_cast<uint64_t>(groups) + group, step = static_cast<uint64_t>(gridDim.x) * groups;
    auto send_for = [&](uint64_t row, int stage) {
        if (row < a.rows) {
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int v = t + i * group_threads;
                if (v >= vectors) continue;
                auto copy = [&](int k, const uint16_t* base, uint64_t ld) {
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(static_cast<uint32_t>(__cvta_generic_to_shared(place(stage, k, i)))),
                                 "l"(reinterpret_cast<const uint4*>(base + row * ld) + v)
                                 : "memory");
                };
                copy(0, a.dy, a.lddy);
                copy(1, a.r, a.ldr);
                if (with_res) copy(2, a.dresidual, a.lddres);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int d = 0; d < kDepth; ++d) send_for(first + d * step, d);
    const float per_col = 1.0f / static_cast<float>(a.cols);
    int stage = 0, turn = 0;
    float rstd_next = first < a.rows ? a.rstd[first] : 0.0f;
    for (uint64_t row = first; row < a.rows; row += step, turn ^= 1) {
        const float rstd = rstd_next;
        rstd_next = row + step < a.rows ? a.rstd[row + step] : 0.0f;
        asm volatile("cp.async.wait_group %0;" ::"n"(kDepth - 1) : "memory");
        uint4 qy[PER], qr[PER], qd[PER];        // kept as they are: unpacked once for the sum and once for dx
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            qy[i] = *place(stage, 0, i);
            qr[i] = *place(stage, 1, i);
            if (with_res) qd[i] = *place(stage, 2, i);
            float y[8], r[8], w[8];
            unpack8(qy[i], y);
            unpack8(qr[i], r);
            unpack8(qw[i], w);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float n = r[e] * rstd;
                dw[i][e] = __fmaf_rn(y[e], n, dw[i][e]);
                sum = __fmaf_rn(y[e] * w[e], n, sum);
            }
        }
        send_for(row + kDepth * step, stage);
        stage = stage + 1 == kDepth ? 0 : stage + 1;
        if (!a.dx) continue;
        sum = warp_sum(sum);
        if (group_warps > 1) {
            if (lane == 0) slots[turn][threadIdx.x >> 5] = sum;
            asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(group_threads) : "memory");
            sum = warp_sum(lane < group_warps ? slots[turn][warp0 + lane] : 0.0f);
        }
        const float mean = sum * per_col;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int v = t + i * group_threads;
            if (v >= vectors) continue;
            float y[8], r[8], w[8], d[8];
            unpack8(qy[i], y);
            unpack8(qr[i], r);
            unpack8(qw[i], w);
#pragma unroll
            for (int e = 0; e < 8; ++e) d[e] = rstd * __fmaf_rn(-r[e] * rstd, mean, y[e] * w[e]);
            if (with_res) {
                float s[8];
                unpack8(qd[i], s);
#pragma unroll
                for (int e = 0; e < 8; ++e) d[e] += s[e];
            }
            reinterpret_cast<uint4*>(a.dx + row * a.lddx)[v] = pack8(d);
        }
    }
    if (!a.dweight) return;
    // the block's groups in order, then one row of partial sums a block
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncthreads();
    float* joined = reinterpret_cast<float*>(dynamic);                  // [groups - 1][cols]
    if (group > 0) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int v = t + i * group_threads;
            if (v >= vectors) continue;
#pragma unroll
            for (int e = 0; e < 8; ++e) joined[(group - 1) * a.cols + v * 8 + e] = dw[i][e];
        }
    }
    __syncthreads();
    if (group == 0) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int v = t + i * group_threads;
            if (v >= vectors) continue;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                for (int g = 1; g < groups; ++g) dw[i][e] += joined[(g - 1) * a.cols + v * 8 + e];
            float4* out = reinterpret_cast<float4*>(a.partial + blockIdx.x * a.cols + v * 8);
            out[0] = make_float4(dw[i][0], dw[i][1], dw[i][2], dw[i][3]);
            out[1] = make_float4(dw[i][4], dw[i][5], dw[i][6], dw[i][7]);
        }
    }
}

// Sums of the blocks' parts, in order: 32 columns a block, each of its 32 warps takes every 32nd part.
constexpr int kFinishSums = 1024;
__global__ void __launch_bounds__(kFinishSums) row_dweight_finish_kernel(const float* partial, int chunks, uint64_t cols, uint16_t* dweight) {
    __shared__ float part[kFinishSums / 32][33];
    after_previous();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint64_t j = blockIdx.x * 32ull + lane;
    float sum = 0.0f;
    if (j < cols) {
#pragma unroll 5
        for (int k = warp; k < chunks; k += kFinishSums / 32) sum += partial[k * cols + j];
    }
    part[warp][lane] = sum;
    __syncthreads();
    sum = warp_sum(part[lane][warp]);                        // column `warp` of the block's
    const uint64_t out = blockIdx.x * 32ull + warp;
    if (lane == 0 && out < cols) dweight[out] = to_bf16(sum);
}

template <int PER, int THREADS>
static unsigned launch_backward_as(const RowBackwardArgs& a, int sm_count, cudaStream_t s) {
    const uint64_t v = a.cols >> 3;
    const int group = static_cast<int>((v + PER * 32 - 1) / (PER * 32) * 32), groups = std::max(1, std::min(kBackwardThreads / group, 15));
    // the places hold the groups' dweight too: 4 cols bytes a group, against 48 kDepth bytes for each 8 columns
    constexpr int place_bytes = kDepth * 3 * PER * 16;
    const uint64_t resident = std::min<uint64_t>(kWeightChunks, (PER > 1 ? 1ull : 2ull) * sm_count);
    const unsigned grid = static_cast<unsigned>(std::min<uint64_t>((a.rows + groups - 1) / groups, resident));
    const collage_status_t st = launch<&row_backward_kernel<PER, THREADS>>(grid, group * groups, 1, place_bytes * group * groups, s, a, group);
    return st == COLLAGE_OK ? grid : 0;
}
// Returns the number of partial rows of dweight, 0 after an error.  Rows of up to 256 columns are a warp's, without barriers;
// longer ones take two vectors a thread (half the barriers and joins of one: 50 against 58 us at 8191 x 4096).  Beyond 8192 columns
// a block of 768 or 1024 threads has too few registers for that and spills 88 and 180 bytes: 4096 x 12288 104 us (3.9 TB/s), 2048 x
// 16384 89 us (3.0), against 262 and 182 element by element (12289 and 16383 columns).
static unsigned launch_backward(const RowBackwardArgs& a, int sm_count, cudaStream_t s) {
    const uint64_t v = a.cols >> 3;
    return v <= 32 ? launch_backward_as<1, 512>(a, sm_count, s)
         : v <= 1024 ? launch_backward_as<2, 512>(a, sm_count, s)
         : v <= 1536 ? launch_backward_as<2, 768>(a, sm_count, s)
                     : launch_backward_as<2, 1024>(a, sm_count, s);
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
    if (x->rows == 0) return COLLAGE_OK;
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
    // (rows without columns go by elements: rstd is NaN, the scale 0)
    bool fit = x->cols && x->cols % 8 == 0 && reinterpret_cast<uintptr_t>(weight) % 16 == 0 && rows_aligned(x, 2, 16);
    for (int i = 0; i < 4; ++i)
        if (others[i]) fit = fit && rows_aligned(others[i], i == 3 ? 1 : 2, i == 3 ? 8 : 16);
    return launch_rows<true>(a, x->rows, fit, dev.sm_count, static_cast<cudaStream_t>(stream));
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
    const bool fit = x->cols % 8 == 0 && rows_aligned(x, 2, 16) && rows_aligned(q, 1, 8);
    return launch_rows<false>(a, x->rows, fit, dev.sm_count, static_cast<cudaStream_t>(stream));
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
    bool fit = dy->cols % 8 == 0 && dy->cols <= 16384 && reinterpret_cast<uintptr_t>(weight) % 16 == 0 && rows_aligned(dy, 2, 16);
    for (const collage_matrix_t* m : others) fit = fit && (!m || rows_aligned(m, 2, 16));
    const unsigned finish_blocks = static_cast<unsigned>((a.cols + 31) / 32);
    if (fit) {
        const unsigned parts = launch_backward(a, dev.sm_count, s);
        if (!parts) return COLLAGE_ERR_CUDA;
        return dweight ? launch<&row_dweight_finish_kernel>(finish_blocks, kFinishSums, 1, 0, s, static_cast<const float*>(a.partial), static_cast<int>(parts), a.cols, a.dweight)
                       : COLLAGE_OK;
    }
    if (dweight) {                            // before dx, which may take dy's place
        uint64_t chunks = (8ull * dev.sm_count + finish_blocks - 1) / finish_blocks;
        chunks = std::min<uint64_t>({chunks, (a.rows + 7) / 8, static_cast<uint64_t>(kWeightChunks)});
        st = launch<&row_dweight_any_kernel>(finish_blocks * chunks, kRowThreads, 1, 0, s, a, static_cast<uint32_t>(chunks));
        if (st == COLLAGE_OK)
            st = launch<&row_dweight_finish_kernel>(finish_blocks, kFinishSums, 1, 0, s, static_cast<const float*>(a.partial), static_cast<int>(chunks), a.cols, a.dweight);
    }
    if (dx && st == COLLAGE_OK) st = launch<&row_backward_any_kernel>(a.rows, kRowThreads, 1, 0, s, a);
    return st;
}

}  // extern "C"

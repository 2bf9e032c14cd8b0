// Norm after a block, its gate and scales, the residual addition and the norm before the next block, in one pass; and its backward pass.
//
//   n = o / sqrt(mean o^2 + eps) * w_post        (o itself without w_post)
//   r = alpha x + beta A(gate) n,                 y = r / sqrt(mean r^2 + eps) * w_pre
// Backward, with nr = r rstd_pre, q = w_pre dy, no = o rstd_post:
//   D = rstd_pre (q - nr mean(q nr)) + dr,        dx = alpha D,     u = beta D
//   h = u A(gate) w_post,                         do = rstd_post (h - no mean(h no))
//   dw_pre = sum dy nr,   dw_post = sum u A no,   dgate = A'(gate) u n  (summed over the rows for a gate of channels)
// where every sum without an index is over the rows.
//
// A row of each array is read once and kept in registers through both of its sums.  Measured at 8191 x 4096 with a gate of channels: forward 48 us
// (5.5 TB/s), backward with all gradients 80 us (5.0 TB/s): memory, and a row's two joins.  With a gate for each token: 2047 x 5120 forward 28
// us (3.7), 45 instructions an element from 14 warps on an SM, and backward 55 us (3.1), one row on an SM at a time.
// As in the residual norm, y belongs to r before r is rounded for the stream.  The backward pass reads the rounded r, or x in its place (FROM_X):
// r is then formed anew, alpha x + (beta A w_post) no, and dw_pre, a sum of dy r, is free of a rounding of each r (relative error at 8191 x 4096
// with a few large columns 0.0016 in place of 0.0022; one rounding of the result is 0.0016).  Same bytes, a few more instructions (38 an
// element in place of 37): backward 84 us in place of 80 at 8191 x 4096, 58 in place of 55 at 2047 x 5120 with a gate for each token.
#include "bulk_pipe.cuh"
#include "ops_common.cuh"

namespace collage {
namespace ops {

struct BlockNormArgs {
    const uint16_t *x, *o, *gate, *post, *pre;
    uint16_t *r, *y;
    uint8_t* y8;
    float *scale, *rstd_post, *rstd_pre;
    uint64_t ldx, ldo, ldg, ldr, ldy, ldy8;      // ldg = 0: one row of gates for all
    uint64_t cols;
    float eps, alpha, beta;
    int activation;
};

// 1 / (1 + exp(-g)) and what it lacks of 1, both to a float's precision wherever g is
__device__ __forceinline__ float2 sigmoids(float g) {
    const float t = __expf(-fabsf(g)), large = __fdividef(1.0f, 1.0f + t), small = t * large;
    return g < 0.0f ? make_float2(small, large) : make_float2(large, small);
}
// A(g), and its derivative; the kind is the same for all threads
__device__ __forceinline__ float gate_value(int kind, float g) {
    if (kind == COLLAGE_GATE_NONE) return g;
    const float s = sigmoids(g).x;
    return kind == COLLAGE_GATE_SIGMOID ? s : g == -INFINITY ? -0.0f : g * s;
}
__device__ __forceinline__ float2 gate_value_and_slope(int kind, float g) {
    if (kind == COLLAGE_GATE_NONE) return make_float2(g, 1.0f);
    const float2 s = sigmoids(g);
    if (kind == COLLAGE_GATE_SIGMOID) return make_float2(s.x, s.x * s.y);
    if (fabsf(g) == INFINITY) return make_float2(g < 0.0f ? -0.0f : g, s.x);
    return make_float2(g * s.x, __fmaf_rn(g * s.x, s.y, s.x));
}
__device__ __forceinline__ float gate_slope(int kind, float g) { return gate_value_and_slope(kind, g).y; }
// The same by way of the smaller one of 1 / (1 + exp(-g)) and what that lacks of 1, which gives both of them to a float's precision.
__device__ __forceinline__ float gate_smaller(int kind, float g) {
    if (kind == COLLAGE_GATE_NONE) return 0.0f;
    const float t = __expf(-fabsf(g));
    return __fdividef(t, 1.0f + t);
}
__device__ __forceinline__ float2 gate_from_smaller(int kind, float g, float small) {
    if (kind == COLLAGE_GATE_NONE) return make_float2(g, 1.0f);
    const float large = 1.0f - small, s = g < 0.0f ? small : large, rest = g < 0.0f ? large : small;
    if (kind == COLLAGE_GATE_SIGMOID) return make_float2(s, s * rest);
    if (fabsf(g) == INFINITY) return make_float2(g < 0.0f ? -0.0f : g, s);
    return make_float2(g * s, __fmaf_rn(g * s, rest, s));
}

constexpr int kBlockThreads = 256;

// One block per row, element by element, the row read again for each stage: any length, stride and alignment.
__global__ void __launch_bounds__(kBlockThreads) block_norm_any_kernel(const __grid_constant__ BlockNormArgs a) {
    __shared__ float slots[kBlockThreads / 32];
    after_previous();
    const uint64_t row = blockIdx.x;
    const uint16_t *x = a.x + row * a.ldx, *o = a.o + row * a.ldo, *gate = a.gate ? a.gate + row * a.ldg : nullptr;
    float fo = 1.0f, rstd_o = 1.0f, fr = 1.0f, rstd_r = 1.0f;
    auto mean_of = [&](auto&& value, float f) {
        float sum = 0.0f;
        for (uint64_t j = threadIdx.x; j < a.cols; j += kBlockThreads) {
            const float v = value(j) * f;
            sum = __fmaf_rn(v, v, sum);
        }
        return block_sum(sum, slots, kBlockThreads / 32) / static_cast<float>(a.cols) + a.eps * f * f;
    };
    auto rstd_of = [&](auto&& value, float& f) {
        float mean = mean_of(value, 1.0f);
        if (!squares_fit(mean)) mean = mean_of(value, f = rescue_factor(mean));
        return 1.0f / sqrtf(mean);
    };
    if (a.post) {
        rstd_o = rstd_of([&](uint64_t j) { return bf16_value(o[j]); }, fo);
        if (a.rstd_post && threadIdx.x == 0) a.rstd_post[row] = fo * rstd_o;
    }
    auto stream = [&](uint64_t j) {
        float n = bf16_value(o[j]);
        if (a.post) n = n * fo * rstd_o * bf16_value(a.post[j]);
        if (gate) n *= gate_value(a.activation, bf16_value(gate[j]));
        return __fmaf_rn(a.alpha, bf16_value(x[j]), a.beta * n);
    };
    if (a.pre) {
        rstd_r = rstd_of(stream, fr);
        if (a.rstd_pre && threadIdx.x == 0) a.rstd_pre[row] = fr * rstd_r;
    }
    auto normed = [&](float r, uint64_t j) { return r * fr * rstd_r * bf16_value(a.pre[j]); };
    float scale = 0.0f;
    if (a.y8) {
        uint32_t most = 0;
        for (uint64_t j = threadIdx.x; j < a.cols; j += kBlockThreads)
            most = max(most, __float_as_uint(normed(stream(j), j)) & 0x7FFFFFFFu);
        most = block_max(most, reinterpret_cast<uint32_t*>(slots), kBlockThreads / 32);
        scale = __uint_as_float(most) / kE4m3Max;
        if (threadIdx.x == 0) a.scale[row] = scale;
    }
    // outputs last, element for element: r may be the array of x or of o, y that of o
    for (uint64_t j = threadIdx.x; j < a.cols; j += kBlockThreads) {
        const float r = stream(j), y = a.pre ? normed(r, j) : 0.0f;
        a.r[row * a.ldr + j] = to_bf16(r);
        if (a.y) a.y[row * a.ldy + j] = to_bf16(y);
        if (a.y8) a.y8[row * a.ldy8 + j] = scale == 0.0f ? 0 : to_e4m3(y / scale);
    }
}

// The same for rows that fit shared memory as floats: each array is read once.  A thread has the same columns in every pass.
constexpr uint64_t kMostStaged = 13 * 1024;          // columns; 16 bytes each in the backward pass
constexpr int kStagedThreads = 512;
// Calls use(j, values of the arrays at column j) for this thread's columns, four at a time with all of their loads sent first.  (Outputs
// may be the arrays of inputs, so that the compiler leaves no load behind a store.)  Absent arrays have zeros.
template <int N, typename Use>
__device__ __forceinline__ void each_column(uint32_t cols, const uint16_t* const (&from)[N], Use&& use) {
    for (uint32_t begin = threadIdx.x; begin < cols; begin += 4 * kStagedThreads) {
        uint16_t raw[4][N];
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int i = 0; i < N; ++i) raw[k][i] = from[i] && begin + k * kStagedThreads < cols ? from[i][begin + k * kStagedThreads] : 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (begin + k * kStagedThreads >= cols) break;
            float values[N];
#pragma unroll
            for (int i = 0; i < N; ++i) values[i] = bf16_value(raw[k][i]);
            use(begin + k * kStagedThreads, values);
        }
    }
}
__global__ void __launch_bounds__(kStagedThreads) block_norm_staged_kernel(const __grid_constant__ BlockNormArgs a, uint64_t rows) {
    __shared__ float slots[kStagedThreads / 32];
    extern __shared__ __align__(16) uint8_t dynamic[];
    float* f = reinterpret_cast<float*>(dynamic);               // [cols]
    after_previous();
    const uint32_t cols = static_cast<uint32_t>(a.cols);
    for (uint64_t row = blockIdx.x; row < rows; row += gridDim.x) {
        const uint16_t *x = a.x + row * a.ldx, *o = a.o + row * a.ldo, *gate = a.gate ? a.gate + row * a.ldg : nullptr;
        // 1 / rms of the values in f from their sum of squares; they come out times a power of two where their squares need one
        auto rstd_of = [&](float sum, float& factor) {
            const float per = static_cast<float>(cols);
            factor = 1.0f;
            float mean = block_sum(sum, slots, kStagedThreads / 32) / per + a.eps;
            if (!squares_fit(mean)) {
                factor = rescue_factor(mean);
                sum = 0.0f;
                for (uint32_t j = threadIdx.x; j < cols; j += kStagedThreads) {
                    f[j] *= factor;
                    sum = __fmaf_rn(f[j], f[j], sum);
                }
                mean = block_sum(sum, slots, kStagedThreads / 32) / per + a.eps * factor * factor;
            }
            return 1.0f / sqrtf(mean);
        };
        float factor, rstd = 1.0f, sum = 0.0f;
        each_column<1>(cols, {o}, [&](uint32_t j, const float (&v)[1]) {
            f[j] = v[0];
            sum = __fmaf_rn(v[0], v[0], sum);
        });
        if (a.post) {
            rstd = rstd_of(sum, factor);
            if (a.rstd_post && threadIdx.x == 0) a.rstd_post[row] = factor * rstd;
        }
        sum = 0.0f;
        each_column<3>(cols, {x, gate, a.post}, [&](uint32_t j, const float (&v)[3]) {
            float n = a.post ? f[j] * rstd * v[2] : f[j];
            if (gate) n *= gate_value(a.activation, v[1]);
            const float r = __fmaf_rn(a.alpha, v[0], a.beta * n);
            f[j] = r;
            a.r[row * a.ldr + j] = to_bf16(r);
            sum = __fmaf_rn(r, r, sum);
        });
        if (!a.pre) continue;
        rstd = rstd_of(sum, factor);
        if (a.rstd_pre && threadIdx.x == 0) a.rstd_pre[row] = factor * rstd;
        uint32_t most = 0;
        each_column<1>(cols, {a.pre}, [&](uint32_t j, const float (&w)[1]) {
            const float y = f[j] * rstd * w[0];
            if (a.y) a.y[row * a.ldy + j] = to_bf16(y);
            f[j] = y;
            most = max(most, __float_as_uint(y) & 0x7FFFFFFFu);
        });
        if (!a.y8) continue;
        const float scale = __uint_as_float(block_max(most, reinterpret_cast<uint32_t*>(slots), kStagedThreads / 32)) / kE4m3Max;
        if (threadIdx.x == 0) a.scale[row] = scale;
#pragma unroll 4
        for (uint32_t j = threadIdx.x; j < cols; j += kStagedThreads) a.y8[row * a.ldy8 + j] = scale == 0.0f ? 0 : to_e4m3(f[j] / scale);
    }
}

// Rows of whole 16-byte vectors, read once and kept in registers: PER vectors a thread, a row by one warp (WARP: four rows a
// block) or by a block of as many warps as it takes.
template <int PER, bool WARP>
__global__ void __launch_bounds__(WARP ? 128 : PER > 2 ? 512 : 1024) block_norm_kernel(const __grid_constant__ BlockNormArgs a, uint64_t rows) {
    __shared__ float slots[32];
    after_previous();
    const uint64_t row = WARP ? blockIdx.x * 4ull + (threadIdx.x >> 5) : blockIdx.x;
    if (WARP && row >= rows) return;
    const int t = WARP ? threadIdx.x & 31 : threadIdx.x, threads = WARP ? 32 : blockDim.x, warps = threads >> 5;
    const int vectors = static_cast<int>(a.cols >> 3);
    const uint4 none = make_uint4(0, 0, 0, 0);
    uint4 qx[PER], qo[PER], qg[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int v = t + i * threads;
        qo[i] = v < vectors ? reinterpret_cast<const uint4*>(a.o + row * a.ldo)[v] : none;
        qx[i] = v < vectors ? reinterpret_cast<const uint4*>(a.x + row * a.ldx)[v] : none;
        if (a.gate) qg[i] = v < vectors ? reinterpret_cast<const uint4*>(a.gate + row * a.ldg)[v] : none;
    }
    float r[PER][8];
    // 1 / rms of the values in r, which come out times a power of two where their squares need one (returned in f)
    auto rstd_of = [&](float& f) {
        f = 1.0f;
#pragma unroll 1
        for (;;) {
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                float part = 0.0f;
#pragma unroll
                for (int e = 0; e < 8; ++e) part = __fmaf_rn(r[i][e], r[i][e], part);
                sum += part;
            }
            const float mean = block_sum(sum, slots, warps) / static_cast<float>(a.cols) + a.eps * f * f;
            if (squares_fit(mean) || f != 1.0f) return 1.0f / sqrtf(mean);
            f = rescue_factor(mean);
#pragma unroll
            for (int i = 0; i < PER; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) r[i][e] *= f;
        }
    };
#pragma unroll
    for (int i = 0; i < PER; ++i) unpack8(qo[i], r[i]);
    if (a.post) {
        uint4 qw[PER];
#pragma unroll
        for (int i = 0; i < PER; ++i) qw[i] = t + i * threads < vectors ? __ldg(reinterpret_cast<const uint4*>(a.post) + t + i * threads) : none;
        float f;
        const float rstd = rstd_of(f);
        if (a.rstd_post && t == 0) a.rstd_post[row] = f * rstd;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            float w[8];
            unpack8(qw[i], w);
#pragma unroll
            for (int e = 0; e < 8; ++e) r[i][e] = r[i][e] * rstd * w[e];
        }
    }
    if (a.gate) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            float g[8];
            unpack8(qg[i], g);
#pragma unroll
            for (int e = 0; e < 8; ++e) r[i][e] *= gate_value(a.activation, g[e]);
        }
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int v = t + i * threads;
        float x[8];
        unpack8(qx[i], x);
#pragma unroll
        for (int e = 0; e < 8; ++e) r[i][e] = v < vectors ? __fmaf_rn(a.alpha, x[e], a.beta * r[i][e]) : 0.0f;
        if (v < vectors) reinterpret_cast<uint4*>(a.r + row * a.ldr)[v] = pack8(r[i]);
    }
    if (!a.pre) return;
    {
        uint4 qw[PER];
#pragma unroll
        for (int i = 0; i < PER; ++i) qw[i] = t + i * threads < vectors ? __ldg(reinterpret_cast<const uint4*>(a.pre) + t + i * threads) : none;
        float f;
        const float rstd = rstd_of(f);
        if (a.rstd_pre && t == 0) a.rstd_pre[row] = f * rstd;
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

// Many rows of whole vectors: a block on each SM walks over rows, one at a time for each group of `group_threads`, two vectors a thread.  What
// the columns are multiplied by is laid out in floats once; a thread sends for its vectors of the next two rows ahead.
constexpr int kRowsDepth = 2, kRowsThreads = 1024;

__global__ void __launch_bounds__(kRowsThreads, 1) block_norm_rows_kernel(const __grid_constant__ BlockNormArgs a, uint64_t rows, int group_threads) {
    constexpr int kArrays = 2, PER = 2;
    __shared__ float slots[2][kRowsThreads / 32];
    __shared__ uint32_t most_slots[kRowsThreads / 32];
    extern __shared__ __align__(16) uint8_t dynamic[];
    after_previous();
    const int groups = blockDim.x / group_threads, group = threadIdx.x / group_threads, t = threadIdx.x % group_threads;
    const int lane = threadIdx.x & 31, group_warps = group_threads >> 5, warp0 = group * group_warps;
    const int vectors = static_cast<int>(a.cols >> 3);
    const uint4 none = make_uint4(0, 0, 0, 0);
    float* post = reinterpret_cast<float*>(dynamic);            // [cols]: beta * post_weight, and A(gate) where it is one of channels
    float* pre = post + a.cols;                                 // [cols]
    uint4* places = reinterpret_cast<uint4*>(dynamic + 8 * a.cols) + threadIdx.x;
    auto place = [&](int stage, int array, int i) { return places + ((stage * kArrays + array) * PER + i) * blockDim.x; };
    for (int d = 0; d < kRowsDepth; ++d)
        for (int k = 0; k < kArrays * PER; ++k) *place(d, 0, k) = none;         // places that no load fills
    for (uint64_t j = threadIdx.x; j < a.cols; j += blockDim.x) {
        float k = a.post ? a.beta * bf16_value(a.post[j]) : a.beta;
        if (a.gate) k *= gate_value(a.activation, bf16_value(a.gate[j]));
        post[j] = k;
        pre[j] = a.pre ? bf16_value(a.pre[j]) : 0.0f;
    }
    const uint64_t first = blockIdx.x * static_cast<uint64_t>(groups) + group, step = static_cast<uint64_t>(gridDim.x) * groups;
    auto send_for = [&](uint64_t row, int stage) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int v = t + i * group_threads;
            if (row >= rows || v >= vectors) continue;
            auto copy = [&](int k, const uint16_t* base, uint64_t ld) {
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(static_cast<uint32_t>(__cvta_generic_to_shared(place(stage, k, i)))),
                             "l"(reinterpret_cast<const uint4*>(base + row * ld) + v)
                             : "memory");
            };
            copy(0, a.o, a.ldo);
            copy(1, a.x, a.ldx);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int d = 0; d < kRowsDepth; ++d) send_for(first + d * step, d);
    __syncthreads();                            // the columns' factors are there
    auto barrier = [&] { asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(group_threads) : "memory"); };
    auto joined = [&](float s, int which) {
        s = warp_sum(s);
        if (group_warps > 1) {
            if (lane == 0) slots[which][threadIdx.x >> 5] = s;
            barrier();
            s = warp_sum(lane < group_warps ? slots[which][warp0 + lane] : 0.0f);
        }
        return s;
    };
    uint64_t f[PER][4];
    // 1 / rms of the values in f, which come out times a power of two where their squares need one (returned in `factor`)
    auto rstd_of = [&](int which, float& factor) {
        auto mean_of = [&](float by) {
            uint64_t sum[PER];
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                sum[i] = mul_pair(f[i][0], f[i][0]);
#pragma unroll
                for (int p = 1; p < 4; ++p) sum[i] = fma_pair(f[i][p], f[i][p], sum[i]);
            }
            return joined(sum_of(sum[0]) + sum_of(sum[1]), which) / static_cast<float>(a.cols) + a.eps * by * by;
        };
        factor = 1.0f;
        float mean = mean_of(1.0f);
        if (!squares_fit(mean)) {
            factor = rescue_factor(mean);
#pragma unroll
            for (int i = 0; i < PER; ++i)
#pragma unroll
                for (int p = 0; p < 4; ++p) f[i][p] = mul_pair(f[i][p], pair_of(factor));
            if (group_warps > 1) barrier();     // (the slots have been read)
            mean = mean_of(factor);
        }
        return 1.0f / sqrtf(mean);
    };
    auto times = [&](const float* k, int v, uint64_t (&g)[4]) {
        const ulonglong2 lo = reinterpret_cast<const ulonglong2*>(k)[2 * v], hi = reinterpret_cast<const ulonglong2*>(k)[2 * v + 1];
        g[0] = mul_pair(g[0], lo.x); g[1] = mul_pair(g[1], lo.y); g[2] = mul_pair(g[2], hi.x); g[3] = mul_pair(g[3], hi.y);
    };
    int stage = 0;
    for (uint64_t row = first; row < rows; row += step) {
        asm volatile("cp.async.wait_group %0;" ::"n"(kRowsDepth - 1) : "memory");
#pragma unroll
        for (int i = 0; i < PER; ++i) unpack_pairs(*place(stage, 0, i), f[i]);
        float factor, rstd = 1.0f;
        if (a.post) {
            rstd = rstd_of(0, factor);
            if (a.rstd_post && t == 0) a.rstd_post[row] = factor * rstd;
        }
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int v = t + i * group_threads;
            uint64_t x[4];
            unpack_pairs(*place(stage, 1, i), x);
#pragma unroll
            for (int p = 0; p < 4; ++p) f[i][p] = mul_pair(f[i][p], pair_of(rstd));
            if (v < vectors) {
                times(post, v, f[i]);
#pragma unroll
                for (int p = 0; p < 4; ++p) f[i][p] = fma_pair(x[p], pair_of(a.alpha), f[i][p]);
                reinterpret_cast<uint4*>(a.r + row * a.ldr)[v] = pack_pairs(f[i]);
            } else {
#pragma unroll
                for (int p = 0; p < 4; ++p) f[i][p] = 0;
            }
        }
        send_for(row + kRowsDepth * step, stage);
        stage = stage + 1 == kRowsDepth ? 0 : stage + 1;
        if (a.pre) {
            rstd = rstd_of(1, factor);
            if (a.rstd_pre && t == 0) a.rstd_pre[row] = factor * rstd;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int v = t + i * group_threads;
                if (v >= vectors) continue;
#pragma unroll
                for (int p = 0; p < 4; ++p) f[i][p] = mul_pair(f[i][p], pair_of(rstd));
                times(pre, v, f[i]);
                if (a.y) reinterpret_cast<uint4*>(a.y + row * a.ldy)[v] = pack_pairs(f[i]);
            }
        }
        if (a.y8) {
            uint32_t most = 0;
#pragma unroll
            for (int i = 0; i < PER; ++i)
#pragma unroll
                for (int p = 0; p < 4; ++p) {
                    const float2 y = floats_of(f[i][p]);
                    if (t + i * group_threads < vectors) most = max(most, max(__float_as_uint(y.x) & 0x7FFFFFFFu, __float_as_uint(y.y) & 0x7FFFFFFFu));
                }
            most = __reduce_max_sync(0xFFFFFFFFu, most);
            if (group_warps > 1) {
                if (lane == 0) most_slots[threadIdx.x >> 5] = most;
                barrier();
                most = __reduce_max_sync(0xFFFFFFFFu, lane < group_warps ? most_slots[warp0 + lane] : 0u);
            }
            const float scale = __uint_as_float(most) / kE4m3Max;
            if (t == 0) a.scale[row] = scale;
            const Divisor by(scale);
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int v = t + i * group_threads;
                if (v >= vectors) continue;
                uint32_t w[2] = {0, 0};
#pragma unroll
                for (int p = 0; p < 4; ++p) {
                    const float2 y = floats_of(f[i][p]);
                    if (by.plain)
                        w[p >> 1] |= pack_e4m3(by.quotient(y.x), by.quotient(y.y)) << (16 * (p & 1));
                    else if (scale != 0.0f)
                        w[p >> 1] |= pack_e4m3(y.x / scale, y.y / scale) << (16 * (p & 1));
                }
                reinterpret_cast<uint2*>(a.y8 + row * a.ldy8)[v] = make_uint2(w[0], w[1]);
            }
        }
        // (of several joins a row, each one's barrier parts the others' slots between rows; one alone needs a second barrier)
        if (group_warps > 1 && (a.post != nullptr) + (a.pre != nullptr) == 1) barrier();
    }
}

static collage_status_t launch_rows(const BlockNormArgs& a, uint64_t rows, int sm_count, cudaStream_t s) {
    const uint64_t v = a.cols >> 3;
    const int group = static_cast<int>((v + 63) / 64 * 32), groups = std::max(1, std::min(kRowsThreads / group, 15));
    const size_t smem = 8 * a.cols + static_cast<size_t>(kRowsDepth) * 2 * 2 * 16 * group * groups;
    const uint64_t grid = std::min<uint64_t>((rows + groups - 1) / groups, static_cast<uint64_t>(sm_count));
    return launch<&block_norm_rows_kernel>(grid, group * groups, 1, smem, s, a, rows, group);
}

// A row's vectors over warps, as in the residual norm: with many rows four vectors a thread, with few rows one.
static collage_status_t launch_block_norm(const BlockNormArgs& a, uint64_t rows, bool vectors_fit, int sm_count, cudaStream_t s) {
    const uint64_t v = a.cols >> 3;
    const bool many = rows > 2ull * sm_count;
    if (!vectors_fit && a.cols <= kMostStaged) return launch<&block_norm_staged_kernel>(std::min<uint64_t>(rows, 4ull * sm_count), kStagedThreads, 1, 4 * a.cols, s, a, rows);
    if (!vectors_fit || v > 4096) return launch<&block_norm_any_kernel>(rows, kBlockThreads, 1, 0, s, a);
    // several rows for each group of threads that walks: 8191 x 4096 48 us against 56, 8191 x 8192 94 against 110; but 8191 x 1024 17 against 15, and 2047 x
    // 5120 with a gate for each token 42 against 28
    if (rows >= 8ull * sm_count && v > 128 && v <= 1024 && !(a.gate && a.ldg)) return launch_rows(a, rows, sm_count, s);
    if (many && v <= 128) {
        const uint64_t grid = (rows + 3) / 4;
        return v <= 32   ? launch<&block_norm_kernel<1, true>>(grid, 128, 1, 0, s, a, rows)
               : v <= 64 ? launch<&block_norm_kernel<2, true>>(grid, 128, 1, 0, s, a, rows)
                         : launch<&block_norm_kernel<4, true>>(grid, 128, 1, 0, s, a, rows);
    }
    const uint64_t per = v > 2048 ? 8 : many ? 4 : v > 1024 ? 2 : 1;
    const int threads = static_cast<int>((v + per * 32 - 1) / (per * 32) * 32);
    return per == 1   ? launch<&block_norm_kernel<1, false>>(rows, threads, 1, 0, s, a, rows)
           : per == 2 ? launch<&block_norm_kernel<2, false>>(rows, threads, 1, 0, s, a, rows)
           : per == 4 ? launch<&block_norm_kernel<4, false>>(rows, threads, 1, 0, s, a, rows)
                      : launch<&block_norm_kernel<8, false>>(rows, threads, 1, 0, s, a, rows);
}

// ------------------------------------------------------------------------------------------------------- backward ---

struct BlockNormBackwardArgs {
    const uint16_t *dy, *dr, *r, *o, *gate, *post, *pre;
    const float *rstd_post, *rstd_pre;
    uint16_t *dx, *dblock, *dgate;        // dgate: a gate for each token; gates of channels come from the sums
    float* partial;                       // [blocks][2][cols]: sum dy nr, and the sum that post_weight and a gate of channels share
    uint64_t lddy, lddr, ldr, ldo, ldg, lddx, lddo, lddg;
    uint64_t rows, cols;
    float alpha, beta;
    int activation, sums;                 // sums: bit 0 for pre_weight, bit 1 for post_weight and gates of channels
    int token_gate;
    int from_x;                           // r is x (and ldr its rows' distance): the stream is formed anew
};

constexpr int kBlockParts = 320;          // blocks whose sums over rows are kept apart
enum { kSumPre = 1, kSumPost = 2 };

// Walks over rows, one block for each, element by element; the sums over its rows are added up in its own part of the workspace.
__global__ void __launch_bounds__(kBlockThreads) block_norm_backward_any_kernel(const __grid_constant__ BlockNormBackwardArgs a) {
    __shared__ float slots[kBlockThreads / 32];
    after_previous();
    float* sum_pre = a.partial + blockIdx.x * 2 * a.cols;
    float* sum_post = sum_pre + a.cols;
    const float per_col = 1.0f / static_cast<float>(a.cols);
    for (uint64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const bool first = row == blockIdx.x;
        const float rstd_r = a.pre ? a.rstd_pre[row] : 0.0f, rstd_o = a.post ? a.rstd_post[row] : 1.0f;
        float mean_r = 0.0f, mean_o = 0.0f;
        auto gate_of = [&](uint64_t j) { return bf16_value(a.gate[row * a.ldg + j]); };
        auto stream = [&](uint64_t j) {
            const float in = bf16_value(a.r[row * a.ldr + j]);
            if (!a.from_x) return in;
            float n = bf16_value(a.o[row * a.ldo + j]);
            if (a.post) n = n * rstd_o * bf16_value(a.post[j]);
            if (a.gate) n *= gate_value(a.activation, gate_of(j));
            return __fmaf_rn(a.alpha, in, a.beta * n);
        };
        if (a.pre) {
            float sum = 0.0f;
            for (uint64_t j = threadIdx.x; j < a.cols; j += kBlockThreads)
                sum = __fmaf_rn(bf16_value(a.dy[row * a.lddy + j]) * bf16_value(a.pre[j]), stream(j) * rstd_r, sum);
            mean_r = block_sum(sum, slots, kBlockThreads / 32) * per_col;
        }
        auto stream_grad = [&](uint64_t j) {
            float d = 0.0f;
            if (a.pre) d = rstd_r * __fmaf_rn(-stream(j) * rstd_r, mean_r, bf16_value(a.dy[row * a.lddy + j]) * bf16_value(a.pre[j]));
            return a.dr ? d + bf16_value(a.dr[row * a.lddr + j]) : d;
        };
        auto gated = [&](uint64_t j, float d) { return a.gate ? a.beta * d * gate_value(a.activation, gate_of(j)) : a.beta * d; };
        if (a.post && a.dblock) {
            float sum = 0.0f;
            for (uint64_t j = threadIdx.x; j < a.cols; j += kBlockThreads)
                sum = __fmaf_rn(gated(j, stream_grad(j)) * bf16_value(a.post[j]), bf16_value(a.o[row * a.ldo + j]) * rstd_o, sum);
            mean_o = block_sum(sum, slots, kBlockThreads / 32) * per_col;
        }
        // outputs last, element for element: they may be the arrays of the gradients that come in
        for (uint64_t j = threadIdx.x; j < a.cols; j += kBlockThreads) {
            const float d = stream_grad(j), n = a.o ? bf16_value(a.o[row * a.ldo + j]) * rstd_o : 0.0f;
            const float du = gated(j, d), w = a.post ? bf16_value(a.post[j]) : 1.0f;
            if (a.sums & kSumPre) {
                const float s = bf16_value(a.dy[row * a.lddy + j]) * (stream(j) * rstd_r);
                sum_pre[j] = first ? s : sum_pre[j] + s;
            }
            if (a.sums & kSumPost) {
                const float s = (a.token_gate ? d * gate_value(a.activation, gate_of(j)) : d) * n;
                sum_post[j] = first ? s : sum_post[j] + s;
            }
            if (a.dgate) a.dgate[row * a.lddg + j] = to_bf16(a.beta * d * n * w * gate_slope(a.activation, gate_of(j)));
            if (a.dx) a.dx[row * a.lddx + j] = to_bf16(a.alpha * d);
            if (a.dblock) a.dblock[row * a.lddo + j] = to_bf16(a.post ? rstd_o * __fmaf_rn(-n, mean_o, du * w) : du);
        }
        __syncthreads();
    }
}

// The same for rows that fit shared memory as floats, with the sums over the block's rows: each array is read once (from x: o and the gate
// twice).  A thread has the same columns in every pass.
__global__ void __launch_bounds__(kStagedThreads) block_norm_backward_staged_kernel(const __grid_constant__ BlockNormBackwardArgs a) {
    __shared__ float slots[kStagedThreads / 32];
    extern __shared__ __align__(16) uint8_t dynamic[];
    const uint32_t cols = static_cast<uint32_t>(a.cols);
    float *d = reinterpret_cast<float*>(dynamic), *n = d + cols, *sum_pre = n + cols, *sum_post = sum_pre + cols;
    after_previous();
    for (uint32_t j = threadIdx.x; j < cols; j += kStagedThreads) sum_pre[j] = sum_post[j] = 0.0f;
    const float per_col = 1.0f / static_cast<float>(cols);
    const bool second = a.post && a.dblock;
    for (uint64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        auto row_of = [&](const uint16_t* p, uint64_t ld) { return p ? p + row * ld : nullptr; };
        const float rstd_r = a.dy ? a.rstd_pre[row] : 0.0f, rstd_o = a.post ? a.rstd_post[row] : 1.0f;
        float mean = 0.0f, sum = 0.0f;
        if (a.dy) {
            auto take = [&](uint32_t j, float dy, float r, float w) {
                const float nr = r * rstd_r, q = dy * w;
                sum_pre[j] = __fmaf_rn(dy, nr, sum_pre[j]);
                sum = __fmaf_rn(q, nr, sum);
                d[j] = q;
                n[j] = nr;
            };
            const uint16_t *dy = row_of(a.dy, a.lddy), *r = row_of(a.r, a.ldr);
            if (a.from_x)
                each_column<6>(cols, {dy, r, a.pre, row_of(a.o, a.ldo), row_of(a.gate, a.ldg), a.post}, [&](uint32_t j, const float (&v)[6]) {
                    float f = a.beta * (a.post ? v[5] : 1.0f);
                    if (a.gate) f *= gate_value(a.activation, v[4]);
                    take(j, v[0], __fmaf_rn(a.alpha, v[1], f * (v[3] * rstd_o)), v[2]);
                });
            else
                each_column<3>(cols, {dy, r, a.pre}, [&](uint32_t j, const float (&v)[3]) { take(j, v[0], v[1], v[2]); });
            mean = block_sum(sum, slots, kStagedThreads / 32) * per_col;
        }
        sum = 0.0f;
        each_column<4>(cols, {row_of(a.dr, a.lddr), row_of(a.o, a.ldo), row_of(a.gate, a.ldg), a.post}, [&](uint32_t j, const float (&in)[4]) {
            const float v = in[0] + (a.dy ? rstd_r * __fmaf_rn(-n[j], mean, d[j]) : 0.0f);
            if (a.dx) a.dx[row * a.lddx + j] = to_bf16(a.alpha * v);
            const float no = in[1] * rstd_o, w = a.beta * (a.post ? in[3] : 1.0f);
            float gated = v;
            if (a.gate) {
                const float2 g = gate_value_and_slope(a.activation, in[2]);
                gated *= g.x;
                if (a.dgate) a.dgate[row * a.lddg + j] = to_bf16(v * w * no * g.y);
            }
            sum_post[j] = __fmaf_rn(a.token_gate ? gated : v, no, sum_post[j]);
            const float h = gated * w;
            sum = __fmaf_rn(h, no, sum);
            if (second) {
                d[j] = h;
                n[j] = no;
            } else if (a.dblock) {
                a.dblock[row * a.lddo + j] = to_bf16(h);
            }
        });
        if (!second) continue;
        mean = block_sum(sum, slots, kStagedThreads / 32) * per_col;
#pragma unroll 4
        for (uint32_t j = threadIdx.x; j < cols; j += kStagedThreads) a.dblock[row * a.lddo + j] = to_bf16(rstd_o * __fmaf_rn(-n[j], mean, d[j]));
    }
    if (!a.sums) return;
    for (uint32_t j = threadIdx.x; j < cols; j += kStagedThreads) {
        a.partial[2ull * blockIdx.x * a.cols + j] = sum_pre[j];
        a.partial[(2ull * blockIdx.x + 1) * a.cols + j] = sum_post[j];
    }
}

// Fault word of this file's waits; collage_pipeline_fault reports it.
static __device__ unsigned int g_block_norm_fault = 0;

// Rows of whole vectors in one pass: a block on each SM walks over rows, one at a time for each group of `group_threads`.  A thread of the
// group brings whole rows into shared memory by bulk copies, several rows ahead, so that the others have nothing to do with loads; each of
// them owns PER vectors of columns, worked on two elements an instruction, and keeps its columns' sums over rows in registers until the end.
constexpr int kMaxGroups = 15, kMaxDepth = 4;
// With a gate for each token a thread keeps its part of post_weight in registers, except from x, which takes it twice a row, where that makes it
// spill: there it is in shared memory, as it came (8191 x 4096 182 us -> 157, 8191 x 1024 54 -> 46, 4096 x 6144 146 -> 143; but 2047 x 5120, for
// which there are registers, 58 -> 60, with a stage less).
template <int PER, bool TOKEN_GATE, bool FROM_X, int THREADS>
constexpr bool kSharesPost = TOKEN_GATE && FROM_X && (PER > 1 || THREADS > 640);

template <int PER, bool TOKEN_GATE, bool FROM_X, int THREADS>
__global__ void __launch_bounds__(THREADS, 1) block_norm_backward_kernel(const __grid_constant__ BlockNormBackwardArgs a, int group_threads, int depth) {
    constexpr int kArrays = TOKEN_GATE ? 5 : 4;
    __shared__ float slots[2][THREADS / 32];
    __shared__ alignas(8) uint64_t full[kMaxGroups * kMaxDepth];
    extern __shared__ __align__(16) uint8_t dynamic[];
    const int groups = blockDim.x / group_threads, group = threadIdx.x / group_threads, t = threadIdx.x % group_threads;
    const int lane = threadIdx.x & 31, group_warps = group_threads >> 5, warp0 = group * group_warps;
    const int vectors = static_cast<int>(a.cols >> 3);
    const uint32_t row_bytes = static_cast<uint32_t>(a.cols * 2), stage_bytes = kArrays * row_bytes;
    if (threadIdx.x == 0) {
        for (int i = 0; i < groups * depth; ++i) pipe::mbar_init(&full[i], 1);
        pipe::mbar_init_fence();
    }
    __syncthreads();
    after_previous();
    uint8_t* stages = dynamic + static_cast<size_t>(group) * depth * stage_bytes;          // of this group: [depth][kArrays] rows
    // what columns are multiplied by, in floats: pre_weight, and beta * post_weight times A(gate) of a gate of channels; with a gate for each
    // token post_weight alone, in bfloat16, or nothing
    float* pre = reinterpret_cast<float*>(dynamic + static_cast<size_t>(groups) * depth * stage_bytes);
    float* post = pre + a.cols;
    const bool second = a.post && a.dblock;
    const uint64_t first = blockIdx.x * static_cast<uint64_t>(groups) + group, step = static_cast<uint64_t>(gridDim.x) * groups;
    const uint32_t sent_bytes = row_bytes * ((a.dy ? 2 : 0) + (a.dr ? 1 : 0) + 1 + (TOKEN_GATE ? 1 : 0));
    bool alive = true;
    auto send_for = [&](uint64_t row, int stage) {             // one thread
        if (row >= a.rows || !alive) return;
        uint8_t* to = stages + stage * stage_bytes;
        uint64_t* bar = &full[group * depth + stage];
        pipe::mbar_arrive_expect_tx(bar, sent_bytes);
        if (a.dy) {
            pipe::bulk_load(to, a.dy + row * a.lddy, row_bytes, bar);
            pipe::bulk_load(to + row_bytes, a.r + row * a.ldr, row_bytes, bar);
        }
        if (a.dr) pipe::bulk_load(to + 2 * row_bytes, a.dr + row * a.lddr, row_bytes, bar);
        pipe::bulk_load(to + 3 * row_bytes, a.o + row * a.ldo, row_bytes, bar);
        if (TOKEN_GATE) pipe::bulk_load(to + 4 * row_bytes, a.gate + row * a.ldg, row_bytes, bar);
    };
    if (t == 0)
        for (int d = 0; d < depth; ++d) send_for(first + d * step, d);
    const uint4 none = make_uint4(0, 0, 0, 0);
    constexpr bool kShared = kSharesPost<PER, TOKEN_GATE, FROM_X, THREADS>, kKept = TOKEN_GATE && !kShared;
    uint4 qpost[kKept ? PER : 1];
    uint64_t sum_pre[PER][4], sum_post[PER][4];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int v = t + i * group_threads;
        if constexpr (kKept) qpost[i] = a.post && v < vectors ? reinterpret_cast<const uint4*>(a.post)[v] : make_uint4(0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u);
#pragma unroll
        for (int p = 0; p < 4; ++p) sum_pre[i][p] = sum_post[i][p] = 0;
    }
    for (uint64_t j = threadIdx.x; j < a.cols; j += blockDim.x) {
        pre[j] = a.pre ? bf16_value(a.pre[j]) : 0.0f;
        if (kShared) reinterpret_cast<uint16_t*>(post)[j] = a.post ? a.post[j] : 0x3F80u;
        if (!TOKEN_GATE) post[j] = a.beta * (a.post ? bf16_value(a.post[j]) : 1.0f) * (a.gate ? gate_value(a.activation, bf16_value(a.gate[j])) : 1.0f);
    }
    __syncthreads();
    auto post_of = [&](int i) {
        if constexpr (kKept)
            return qpost[i];
        else
            return reinterpret_cast<const uint4*>(post)[min(t + i * group_threads, vectors - 1)];
    };
    const float per_col = 1.0f / static_cast<float>(a.cols);
    auto barrier = [&] {
        if (group_warps > 1)
            asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(group_threads) : "memory");
        else
            __syncwarp();
    };
    // over the group; the two sums of a row have slots of their own, so that one barrier each is enough
    auto joined = [&](float s, int which) {
        s = warp_sum(s);
        if (group_warps > 1) {
            if (lane == 0) slots[which][threadIdx.x >> 5] = s;
            barrier();
            s = warp_sum(lane < group_warps ? slots[which][warp0 + lane] : 0.0f);
        }
        return s;
    };
    int stage = 0;
    uint32_t phase = 0;
    uint64_t gave_up = a.rows;
    float rstd_r = a.dy && first < a.rows ? a.rstd_pre[first] : 0.0f, rstd_o = a.post && first < a.rows ? a.rstd_post[first] : 1.0f;
    for (uint64_t row = first; row < a.rows; row += step) {
        const float next_r = a.dy && row + step < a.rows ? a.rstd_pre[row + step] : 0.0f, next_o = a.post && row + step < a.rows ? a.rstd_post[row + step] : 1.0f;
        // (after a wait that was given up all go on together, without waiting: the barriers below are for all of the group)
        if (alive && !pipe::mbar_wait(&full[group * depth + stage], phase, 400, &g_block_norm_fault)) {
            alive = false;
            gave_up = row;
        }
        uint8_t* here = stages + stage * stage_bytes;
        auto vector = [&](int array, int i) {
            const int v = t + i * group_threads;
            return v < vectors ? reinterpret_cast<const uint4*>(here + array * row_bytes)[v] : none;
        };
        auto factors = [&](const float* k, int i, uint64_t (&w)[4]) {
            const int v = min(t + i * group_threads, vectors - 1);          // (the vectors of columns that are not there are zeros)
            const ulonglong2 lo = reinterpret_cast<const ulonglong2*>(k)[2 * v], hi = reinterpret_cast<const ulonglong2*>(k)[2 * v + 1];
            w[0] = lo.x; w[1] = lo.y; w[2] = hi.x; w[3] = hi.y;
        };
        uint64_t n[PER][4], d[PER][4];          // n of the stream, then of the block; the gradient on its way from y to the block
        auto normed_block = [&](int i, uint64_t (&to)[4]) {
            unpack_pairs(vector(3, i), to);
#pragma unroll
            for (int p = 0; p < 4; ++p) to[p] = mul_pair(to[p], pair_of(rstd_o));
        };
        float mean = 0.0f;
        if (FROM_X || a.dy) {
            uint64_t sum = 0;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                uint64_t dy[4], w[4];
                unpack_pairs(vector(0, i), dy);
                unpack_pairs(vector(1, i), n[i]);
                if constexpr (FROM_X) {
                    uint64_t no[4];
                    normed_block(i, no);
                    if constexpr (TOKEN_GATE) {
                        uint64_t g[4];
                        unpack_pairs(vector(4, i), g);
                        unpack_pairs(post_of(i), w);
                        float small[8];         // for the second pass, in the place of this thread's dy and x
#pragma unroll
                        for (int p = 0; p < 4; ++p) {
                            const float2 gf = floats_of(g[p]);
                            small[2 * p] = gate_smaller(a.activation, gf.x);
                            small[2 * p + 1] = gate_smaller(a.activation, gf.y);
                            w[p] = mul_pair(mul_pair(w[p], pair_of(a.beta)),
                                            pair_of(gate_from_smaller(a.activation, gf.x, small[2 * p]).x, gate_from_smaller(a.activation, gf.y, small[2 * p + 1]).x));
                        }
                        if (const int v = t + i * group_threads; v < vectors) {
                            reinterpret_cast<float4*>(here)[v] = make_float4(small[0], small[1], small[2], small[3]);
                            reinterpret_cast<float4*>(here + row_bytes)[v] = make_float4(small[4], small[5], small[6], small[7]);
                        }
                    } else {
                        factors(post, i, w);
                    }
#pragma unroll
                    for (int p = 0; p < 4; ++p) n[i][p] = fma_pair(n[i][p], pair_of(a.alpha), mul_pair(no[p], w[p]));
                }
                factors(pre, i, w);
#pragma unroll
                for (int p = 0; p < 4; ++p) {
                    n[i][p] = mul_pair(n[i][p], pair_of(rstd_r));
                    sum_pre[i][p] = fma_pair(dy[p], n[i][p], sum_pre[i][p]);
                    d[i][p] = mul_pair(dy[p], w[p]);
                    sum = fma_pair(d[i][p], n[i][p], sum);
                }
            }
            if (TOKEN_GATE && FROM_X) pipe::fence_async_smem();        // (what was written to the stage, before a copy may come over it)
            mean = joined(sum_of(sum), 0) * per_col;
        }
        uint64_t sum = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int v = t + i * group_threads;
            uint64_t dr[4] = {0, 0, 0, 0};
            if (a.dr) unpack_pairs(vector(2, i), dr);
#pragma unroll
            for (int p = 0; p < 4; ++p) d[i][p] = a.dy ? fma_pair(fma_pair(n[i][p], pair_of(-mean), d[i][p]), pair_of(rstd_r), dr[p]) : dr[p];
            if (a.dx && v < vectors) {
                uint64_t dx[4];
#pragma unroll
                for (int p = 0; p < 4; ++p) dx[p] = mul_pair(d[i][p], pair_of(a.alpha));
                reinterpret_cast<uint4*>(a.dx + row * a.lddx)[v] = pack_pairs(dx);
            }
            uint64_t w[4];
            normed_block(i, n[i]);
            if (TOKEN_GATE) {
                uint64_t g[4];
                unpack_pairs(vector(4, i), g);
                unpack_pairs(post_of(i), w);
                float parts[8];
                if constexpr (FROM_X) {
                    const uint4 lo = vector(0, i), hi = vector(1, i);
                    const uint32_t words[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
                    for (int e = 0; e < 8; ++e) parts[e] = __uint_as_float(words[e]);
                }
#pragma unroll
                for (int p = 0; p < 4; ++p) {
                    const float2 gf = floats_of(g[p]);
                    float2 lo, hi;
                    if constexpr (FROM_X) {
                        lo = gate_from_smaller(a.activation, gf.x, parts[2 * p]);
                        hi = gate_from_smaller(a.activation, gf.y, parts[2 * p + 1]);
                    } else {
                        lo = gate_value_and_slope(a.activation, gf.x);
                        hi = gate_value_and_slope(a.activation, gf.y);
                    }
                    const uint64_t gated = mul_pair(d[i][p], pair_of(lo.x, hi.x));
                    sum_post[i][p] = fma_pair(gated, n[i][p], sum_post[i][p]);
                    w[p] = mul_pair(w[p], pair_of(a.beta));
                    g[p] = mul_pair(mul_pair(mul_pair(d[i][p], w[p]), n[i][p]), pair_of(lo.y, hi.y));
                    d[i][p] = mul_pair(gated, w[p]);
                }
                if (a.dgate && v < vectors) reinterpret_cast<uint4*>(a.dgate + row * a.lddg)[v] = pack_pairs(g);
            } else {
                factors(post, i, w);
#pragma unroll
                for (int p = 0; p < 4; ++p) {
                    sum_post[i][p] = fma_pair(d[i][p], n[i][p], sum_post[i][p]);
                    d[i][p] = mul_pair(d[i][p], w[p]);
                }
            }
            if (second) {
#pragma unroll
                for (int p = 0; p < 4; ++p) sum = fma_pair(d[i][p], n[i][p], sum);
            }
        }
        if (second) {
            mean = joined(sum_of(sum), 1) * per_col;
#pragma unroll
            for (int i = 0; i < PER; ++i)
#pragma unroll
                for (int p = 0; p < 4; ++p) d[i][p] = mul_pair(fma_pair(n[i][p], pair_of(-mean), d[i][p]), pair_of(rstd_o));
        }
        // All of the group has read the stage: behind the second sum's barrier, or, without one, behind this.  (It parts the slots of one
        // row's only sum from the next one's, too; of two, each one's barrier does that for the other.)
        if (!(second && a.dy) || group_warps == 1) barrier();
        if (t == 0) send_for(row + depth * step, stage);
        if (a.dblock) {
#pragma unroll
            for (int i = 0; i < PER; ++i)
                if (t + i * group_threads < vectors) reinterpret_cast<uint4*>(a.dblock + row * a.lddo)[t + i * group_threads] = pack_pairs(d[i]);
        }
        if (++stage == depth) { stage = 0; phase ^= 1; }
        rstd_r = next_r;
        rstd_o = next_o;
    }
    if (!alive && t == 0)                       // the copies that are still under way
        for (uint64_t row = gave_up, it = (gave_up - first) / step, end = it + depth; row < a.rows && it < end; row += step, ++it)
            pipe::mbar_wait(&full[group * depth + it % depth], it / depth & 1u, 401, &g_block_norm_fault);
    if (!a.sums) return;
    // the block's groups in order, then one row of partial sums a block
    __syncthreads();
    ulonglong2* shared_sums = reinterpret_cast<ulonglong2*>(dynamic);         // [groups][PER][group_threads][4]: pairs of both sums
    auto part = [&](int g, int i) { return shared_sums + ((static_cast<size_t>(g) * PER + i) * group_threads + t) * 4; };
    if (group > 0) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            ulonglong2* to = part(group, i);
            to[0] = make_ulonglong2(sum_pre[i][0], sum_pre[i][1]);
            to[1] = make_ulonglong2(sum_pre[i][2], sum_pre[i][3]);
            to[2] = make_ulonglong2(sum_post[i][0], sum_post[i][1]);
            to[3] = make_ulonglong2(sum_post[i][2], sum_post[i][3]);
        }
    }
    __syncthreads();
    if (group > 0) return;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int v = t + i * group_threads;
        if (v >= vectors) continue;
        for (int g = 1; g < groups; ++g) {
            const ulonglong2* from = part(g, i);
            sum_pre[i][0] = add_pair(sum_pre[i][0], from[0].x); sum_pre[i][1] = add_pair(sum_pre[i][1], from[0].y);
            sum_pre[i][2] = add_pair(sum_pre[i][2], from[1].x); sum_pre[i][3] = add_pair(sum_pre[i][3], from[1].y);
            sum_post[i][0] = add_pair(sum_post[i][0], from[2].x); sum_post[i][1] = add_pair(sum_post[i][1], from[2].y);
            sum_post[i][2] = add_pair(sum_post[i][2], from[3].x); sum_post[i][3] = add_pair(sum_post[i][3], from[3].y);
        }
        ulonglong2* out = reinterpret_cast<ulonglong2*>(a.partial + 2ull * blockIdx.x * a.cols + v * 8);
        out[0] = make_ulonglong2(sum_pre[i][0], sum_pre[i][1]);
        out[1] = make_ulonglong2(sum_pre[i][2], sum_pre[i][3]);
        out = reinterpret_cast<ulonglong2*>(a.partial + (2ull * blockIdx.x + 1) * a.cols + v * 8);
        out[0] = make_ulonglong2(sum_post[i][0], sum_post[i][1]);
        out[1] = make_ulonglong2(sum_post[i][2], sum_post[i][3]);
    }
}

template <int PER, bool TOKEN_GATE, bool FROM_X, int THREADS>
static collage_status_t launch_block_backward_as(const BlockNormBackwardArgs& a, unsigned* parts, int sm_count, cudaStream_t s) {
    const uint64_t v = a.cols >> 3;
    const int group = static_cast<int>((v + PER * 32 - 1) / (PER * 32) * 32), most = std::max(1, std::min(THREADS / group, kMaxGroups));
    // few rows: as many groups as give every SM some
    const int groups = static_cast<int>(std::max<uint64_t>(1, std::min<uint64_t>(most, (a.rows + sm_count - 1) / sm_count)));
    const size_t row = (TOKEN_GATE ? 5 : 4) * 2 * a.cols, factors = (!TOKEN_GATE ? 8 : kSharesPost<PER, TOKEN_GATE, FROM_X, THREADS> ? 6 : 4) * a.cols;
    const int depth = static_cast<int>(std::min<size_t>(kMaxDepth, (224 * 1024 - factors) / (row * groups)));
    // the stages hold the groups' sums in the end: 64 PER bytes a thread
    const size_t smem = std::max<size_t>(depth * row * groups, 64ull * PER * group * groups) + factors;
    *parts = static_cast<unsigned>(std::min<uint64_t>((a.rows + groups - 1) / groups, static_cast<uint64_t>(sm_count)));
    return launch<&block_norm_backward_kernel<PER, TOKEN_GATE, FROM_X, THREADS>>(*parts, group * groups, 1, smem, s, a, group, depth);
}
// Rows of up to 256 columns are a warp's, without barriers; longer ones take two vectors a thread, half the joins of one.  Of rows that leave
// many of 512 threads idle that way (and a second row has no registers) one vector a thread is faster: 2047 x 5120 with a gate for each
// token 55 us against 76, 4096 x 6144 106 against 138, 8191 x 5120 without 119 against 128, but 8191 x 6144 141 against 133.
template <bool TOKEN_GATE, bool FROM_X>
static collage_status_t launch_block_backward(const BlockNormBackwardArgs& a, unsigned* parts, int sm_count, cudaStream_t s) {
    if (a.cols <= 256) return launch_block_backward_as<1, TOKEN_GATE, FROM_X, 512>(a, parts, sm_count, s);
    if (a.cols > 4096 && a.cols <= 5120) return launch_block_backward_as<1, TOKEN_GATE, FROM_X, 640>(a, parts, sm_count, s);
    if (TOKEN_GATE && a.cols > 5120 && a.cols <= 6144) return launch_block_backward_as<1, TOKEN_GATE, FROM_X, 768>(a, parts, sm_count, s);
    return launch_block_backward_as<2, TOKEN_GATE, FROM_X, 512>(a, parts, sm_count, s);
}

// The blocks' parts added up in order: 32 columns a block, each of its 32 warps takes every 32nd part.  From the shared sum
// S = beta sum D n: dpost = A S and dgate = A' w S for a gate of channels; otherwise the gate is in the sum and dpost = S.
struct BlockNormFinishArgs {
    const float* partial;
    const uint16_t *gate, *post;          // gate: of channels, or null
    uint16_t *dpre, *dpost, *dgate;
    uint64_t cols;
    float beta;
    int parts, activation;
};
constexpr int kBlockFinish = 1024;
__global__ void __launch_bounds__(kBlockFinish) block_norm_finish_kernel(const __grid_constant__ BlockNormFinishArgs a, uint32_t column_blocks, int first_kind) {
    __shared__ float part[kBlockFinish / 32][33];
    after_previous();
    const int kind = blockIdx.x / column_blocks + first_kind;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint64_t begin = (blockIdx.x % column_blocks) * 32ull, j = begin + lane;
    float sum = 0.0f;
    if (j < a.cols) {
#pragma unroll 5
        for (int k = warp; k < a.parts; k += kBlockFinish / 32) sum += a.partial[(2ull * k + kind) * a.cols + j];
    }
    part[warp][lane] = sum;
    __syncthreads();
    sum = warp_sum(part[lane][warp]);                        // column `warp` of the block's
    const uint64_t out = begin + warp;
    if (lane || out >= a.cols) return;
    if (kind == 0) {
        a.dpre[out] = to_bf16(sum);
        return;
    }
    sum *= a.beta;
    const float g = a.gate ? bf16_value(a.gate[out]) : 1.0f;
    if (a.dpost) a.dpost[out] = to_bf16(a.gate ? gate_value(a.activation, g) * sum : sum);
    if (a.dgate) a.dgate[out] = to_bf16((a.post ? bf16_value(a.post[out]) : 1.0f) * sum * gate_slope(a.activation, g));
}

}  // namespace ops
}  // namespace collage

using namespace collage;
using namespace collage::ops;

namespace {
// A gate is absent (no data), one row for all, or a row for each.
bool has_gate(const collage_block_norm_t* in) { return in->gate.data != nullptr; }
bool gate_of_channels(const collage_block_norm_t* in) { return has_gate(in) && in->gate.rows == 1 && in->block.rows != 1; }

collage_status_t check_block_norm(const collage_block_norm_t* in, uint64_t rows, uint64_t cols) {
    auto scale_fits = [](double v) { return std::isfinite(v) && std::isfinite(static_cast<float>(v)); };
    if (!scale_fits(in->residual_scale) || !scale_fits(in->block_scale) || !(scale_fits(in->eps) && in->eps >= 0.0)) return COLLAGE_ERR_ARG;
    if (in->activation < COLLAGE_GATE_NONE || in->activation > COLLAGE_GATE_SILU) return COLLAGE_ERR_ARG;
    if (has_gate(in) && (in->gate.cols != cols || (in->gate.rows != 1 && in->gate.rows != rows))) return COLLAGE_ERR_ARG;
    if (reinterpret_cast<uintptr_t>(in->post_weight) % 2 || reinterpret_cast<uintptr_t>(in->pre_weight) % 2) return COLLAGE_ERR_ARG;
    return has_gate(in) ? check_matrix(&in->gate, 2) : COLLAGE_OK;
}
bool aligned(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }
}  // namespace

namespace collage {
cudaError_t read_clear_block_norm_fault(unsigned int* out) {
    const unsigned int zero = 0;
    const cudaError_t e = cudaMemcpyFromSymbol(out, g_block_norm_fault, sizeof *out);
    return e != cudaSuccess || *out == 0 ? e : cudaMemcpyToSymbol(g_block_norm_fault, &zero, sizeof zero);
}
}  // namespace collage

extern "C" {

collage_status_t collage_block_norm(const collage_block_norm_t* in, const collage_matrix_t* x, const collage_matrix_t* r, const collage_matrix_t* y,
                                    const collage_matrix_t* y8, float* y8_scale, float* rstd_post, float* rstd_pre, void* stream) {
    if (!in || !x || !r || (y8 && !y8_scale && x->rows)) return COLLAGE_ERR_NULL;
    if (!in->pre_weight && x->cols && (y || y8)) return COLLAGE_ERR_NULL;
    if ((y8_scale && !y8) || (rstd_post && !in->post_weight && x->cols) || (rstd_pre && !in->pre_weight && x->cols)) return COLLAGE_ERR_ARG;
    const collage_matrix_t* all[5] = {x, &in->block, r, y, y8};
    collage_status_t st = COLLAGE_OK;
    for (int i = 0; i < 5 && st == COLLAGE_OK; ++i)
        if (all[i]) st = !same_shape(x, all[i]) ? COLLAGE_ERR_ARG : check_matrix(all[i], i == 4 ? 1 : 2);
    if (st == COLLAGE_OK) st = check_block_norm(in, x->rows, x->cols);
    if (st != COLLAGE_OK) return st;
    if (reinterpret_cast<uintptr_t>(y8_scale) % 4 || reinterpret_cast<uintptr_t>(rstd_post) % 4 || reinterpret_cast<uintptr_t>(rstd_pre) % 4)
        return COLLAGE_ERR_ARG;
    AliasCheck alias;
    const int ix = alias.add(span_of(x, 2), false), io = alias.add(span_of(&in->block, 2), false);
    if (has_gate(in)) alias.add(span_of(&in->gate, 2), false);
    alias.add(span_of(in->post_weight, 2 * x->cols), false);
    alias.add(span_of(in->pre_weight, 2 * x->cols), false);
    const int ir = alias.add(span_of(r, 2), true), iy = y ? alias.add(span_of(y, 2), true) : -1;
    if (y8) alias.add(span_of(y8, 1), true);
    if (y8_scale) alias.add(span_of(y8_scale, 4 * x->rows), true);
    if (rstd_post) alias.add(span_of(rstd_post, 4 * x->rows), true);
    if (rstd_pre) alias.add(span_of(rstd_pre, 4 * x->rows), true);
    const int pairs[3][2] = {{ir, ix}, {ir, io}, {iy, io}};
    if (alias.clash(pairs)) return COLLAGE_ERR_ALIAS;
    DeviceInfo dev;
    if ((st = current_device(&dev)) != COLLAGE_OK) return st;
    if (x->rows == 0) return COLLAGE_OK;
    BlockNormArgs a = {};
    a.x = static_cast<const uint16_t*>(x->data);
    a.ldx = x->ld;
    a.o = static_cast<const uint16_t*>(in->block.data);
    a.ldo = in->block.ld;
    if (has_gate(in)) { a.gate = static_cast<const uint16_t*>(in->gate.data); a.ldg = in->gate.rows == 1 ? 0 : in->gate.ld; }
    a.post = static_cast<const uint16_t*>(in->post_weight);
    a.pre = static_cast<const uint16_t*>(in->pre_weight);
    a.r = static_cast<uint16_t*>(r->data);
    a.ldr = r->ld;
    if (y) { a.y = static_cast<uint16_t*>(y->data); a.ldy = y->ld; }
    if (y8) { a.y8 = static_cast<uint8_t*>(y8->data); a.ldy8 = y8->ld; a.scale = y8_scale; }
    a.rstd_post = rstd_post;
    a.rstd_pre = rstd_pre;
    a.cols = x->cols;
    a.eps = static_cast<float>(in->eps);
    a.alpha = static_cast<float>(in->residual_scale);
    a.beta = static_cast<float>(in->block_scale);
    a.activation = in->activation;
    if (x->cols == 0) {                        // no values: scales of 0, no rms
        cudaStream_t s = static_cast<cudaStream_t>(stream);
        if (y8_scale && cudaMemsetAsync(y8_scale, 0, 4 * x->rows, s) != cudaSuccess) return COLLAGE_ERR_CUDA;
        for (float* p : {rstd_post, rstd_pre})
            if (p && cudaMemsetAsync(p, 0xFF, 4 * x->rows, s) != cudaSuccess) return COLLAGE_ERR_CUDA;      // (a NaN)
        return COLLAGE_OK;
    }
    bool fit = x->cols % 8 == 0 && aligned(a.post) && aligned(a.pre) && (!a.gate || rows_aligned(&in->gate, 2, 16));
    for (int i = 0; i < 5; ++i)
        if (all[i]) fit = fit && rows_aligned(all[i], i == 4 ? 1 : 2, i == 4 ? 8 : 16);
    return launch_block_norm(a, x->rows, fit, dev.sm_count, static_cast<cudaStream_t>(stream));
}

size_t collage_block_norm_workspace_bytes(uint64_t cols) { return static_cast<size_t>(kBlockParts) * 8 * cols; }

}  // extern "C"

// Both entry points; `r` is x if from_x.
static collage_status_t block_norm_backward(const collage_block_norm_t* in, bool from_x, const collage_matrix_t* dy, const collage_matrix_t* dr,
                                            const collage_matrix_t* r, const float* rstd_post, const float* rstd_pre, const collage_matrix_t* dx,
                                            const collage_matrix_t* dblock, const collage_matrix_t* dgate, void* dpost_weight, void* dpre_weight,
                                            void* workspace, size_t workspace_bytes, void* stream) {
    if (!in) return COLLAGE_ERR_NULL;
    const collage_matrix_t* o = &in->block;
    const uint64_t rows = o->rows, cols = o->cols;
    if (cols && ((!dy && !dr) || (!dx && !dblock && !dgate && !dpost_weight && !dpre_weight))) return COLLAGE_ERR_NULL;
    if (cols && rows && ((dy && (!r || !rstd_pre || !in->pre_weight)) || (in->post_weight && !rstd_post))) return COLLAGE_ERR_NULL;
    if ((dpre_weight && !dy) || (dpost_weight && !in->post_weight) || (dgate && !has_gate(in))) return COLLAGE_ERR_ARG;
    const collage_matrix_t* all[6] = {o, dy, dr, r, dx, dblock};
    collage_status_t st = COLLAGE_OK;
    for (int i = 0; i < 6 && st == COLLAGE_OK; ++i)
        if (all[i]) st = !same_shape(o, all[i]) ? COLLAGE_ERR_ARG : check_matrix(all[i], 2);
    if (st == COLLAGE_OK) st = check_block_norm(in, rows, cols);
    if (st == COLLAGE_OK && dgate) st = !same_shape(&in->gate, dgate) ? COLLAGE_ERR_ARG : check_matrix(dgate, 2);
    if (st != COLLAGE_OK) return st;
    if (reinterpret_cast<uintptr_t>(rstd_post) % 4 || reinterpret_cast<uintptr_t>(rstd_pre) % 4 || reinterpret_cast<uintptr_t>(dpost_weight) % 2 ||
        reinterpret_cast<uintptr_t>(dpre_weight) % 2)
        return COLLAGE_ERR_ARG;
    const bool channels = gate_of_channels(in), channel_grad = dgate && channels;
    const int sums = (dpre_weight ? kSumPre : 0) | (dpost_weight || channel_grad ? kSumPost : 0);
    const size_t need = collage_block_norm_workspace_bytes(cols);
    if (sums && need && (!workspace || workspace_bytes < need || !aligned(workspace))) return COLLAGE_ERR_WORKSPACE;
    AliasCheck alias;
    alias.add(span_of(o, 2), false);
    if (has_gate(in)) alias.add(span_of(&in->gate, 2), false);
    alias.add(span_of(in->post_weight, 2 * cols), false);
    alias.add(span_of(in->pre_weight, 2 * cols), false);
    const int idy = dy ? alias.add(span_of(dy, 2), false) : -1, idr = dr ? alias.add(span_of(dr, 2), false) : -1;
    if (dy && r) alias.add(span_of(r, 2), false);
    if (rstd_post) alias.add(span_of(rstd_post, 4 * rows), false);
    if (rstd_pre) alias.add(span_of(rstd_pre, 4 * rows), false);
    const int idx = dx ? alias.add(span_of(dx, 2), true) : -1, ido = dblock ? alias.add(span_of(dblock, 2), true) : -1;
    if (dgate) alias.add(span_of(dgate, 2), true);
    if (dpost_weight) alias.add(span_of(dpost_weight, 2 * cols), true);
    if (dpre_weight) alias.add(span_of(dpre_weight, 2 * cols), true);
    if (sums) alias.add(span_of(workspace, need), true);
    const int pairs[4][2] = {{idx, idy}, {idx, idr}, {ido, idy}, {ido, idr}};
    if (alias.clash(pairs)) return COLLAGE_ERR_ALIAS;
    DeviceInfo dev;
    if ((st = current_device(&dev)) != COLLAGE_OK) return st;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (cols == 0) return COLLAGE_OK;
    if (rows == 0) {                           // sums over nothing
        for (void* p : {dpost_weight, dpre_weight, channel_grad ? dgate->data : nullptr})
            if (p && cudaMemsetAsync(p, 0, 2 * cols, s) != cudaSuccess) return COLLAGE_ERR_CUDA;
        return COLLAGE_OK;
    }
    BlockNormBackwardArgs a = {};
    auto set = [](const collage_matrix_t* m, const uint16_t*& p, uint64_t& ld) { if (m) { p = static_cast<const uint16_t*>(m->data); ld = m->ld; } };
    auto set_out = [](const collage_matrix_t* m, uint16_t*& p, uint64_t& ld) { if (m) { p = static_cast<uint16_t*>(m->data); ld = m->ld; } };
    set(dr, a.dr, a.lddr);
    if (dy) {
        set(dy, a.dy, a.lddy);
        set(r, a.r, a.ldr);
        a.pre = static_cast<const uint16_t*>(in->pre_weight);
        a.rstd_pre = rstd_pre;
        a.from_x = from_x;
    }
    set(o, a.o, a.ldo);
    if (has_gate(in)) { a.gate = static_cast<const uint16_t*>(in->gate.data); a.ldg = in->gate.rows == 1 ? 0 : in->gate.ld; }
    a.token_gate = has_gate(in) && !channels;
    a.post = static_cast<const uint16_t*>(in->post_weight);
    a.rstd_post = rstd_post;
    set_out(dx, a.dx, a.lddx);
    set_out(dblock, a.dblock, a.lddo);
    if (!channels) set_out(dgate, a.dgate, a.lddg);
    a.partial = static_cast<float*>(workspace);
    a.rows = rows;
    a.cols = cols;
    a.alpha = static_cast<float>(in->residual_scale);
    a.beta = static_cast<float>(in->block_scale);
    a.activation = in->activation;
    a.sums = sums;
    bool fit = cols % 8 == 0 && cols <= 8192 && aligned(a.post) && aligned(a.pre) && (!a.gate || rows_aligned(&in->gate, 2, 16)) &&
               (!a.dgate || rows_aligned(dgate, 2, 16));
    for (const collage_matrix_t* m : all) fit = fit && (!m || rows_aligned(m, 2, 16));
    unsigned parts = static_cast<unsigned>(std::min<uint64_t>({rows, static_cast<uint64_t>(kBlockParts), 2ull * dev.sm_count}));
    if (!fit && cols <= kMostStaged)
        st = launch<&block_norm_backward_staged_kernel>(parts, kStagedThreads, 1, 16 * cols, s, a);
    else if (!fit)
        st = launch<&block_norm_backward_any_kernel>(parts, kBlockThreads, 1, 0, s, a);
    else if (a.from_x)
        st = a.token_gate ? launch_block_backward<true, true>(a, &parts, dev.sm_count, s) : launch_block_backward<false, true>(a, &parts, dev.sm_count, s);
    else
        st = a.token_gate ? launch_block_backward<true, false>(a, &parts, dev.sm_count, s) : launch_block_backward<false, false>(a, &parts, dev.sm_count, s);
    if (st != COLLAGE_OK || !sums) return st;
    BlockNormFinishArgs f = {};
    f.partial = a.partial;
    f.gate = channels ? a.gate : nullptr;
    f.post = a.post;
    f.dpre = static_cast<uint16_t*>(dpre_weight);
    f.dpost = static_cast<uint16_t*>(dpost_weight);
    f.dgate = channel_grad ? static_cast<uint16_t*>(dgate->data) : nullptr;
    f.cols = cols;
    f.beta = a.beta;
    f.parts = static_cast<int>(parts);
    f.activation = in->activation;
    const uint32_t column_blocks = static_cast<uint32_t>((cols + 31) / 32);
    const int kinds = (sums & kSumPre ? 1 : 0) + (sums & kSumPost ? 1 : 0);
    return launch<&block_norm_finish_kernel>(static_cast<uint64_t>(column_blocks) * kinds, kBlockFinish, 1, 0, s, f, column_blocks, sums & kSumPre ? 0 : 1);
}

extern "C" {

collage_status_t collage_block_norm_backward(const collage_block_norm_t* in, const collage_matrix_t* dy, const collage_matrix_t* dr,
                                             const collage_matrix_t* r, const float* rstd_post, const float* rstd_pre,
                                             const collage_matrix_t* dx, const collage_matrix_t* dblock, const collage_matrix_t* dgate,
                                             void* dpost_weight, void* dpre_weight, void* workspace, size_t workspace_bytes, void* stream) {
    return block_norm_backward(in, false, dy, dr, r, rstd_post, rstd_pre, dx, dblock, dgate, dpost_weight, dpre_weight, workspace, workspace_bytes, stream);
}

collage_status_t collage_block_norm_backward_from_x(const collage_block_norm_t* in, const collage_matrix_t* dy, const collage_matrix_t* dr,
                                                    const collage_matrix_t* x, const float* rstd_post, const float* rstd_pre,
                                                    const collage_matrix_t* dx, const collage_matrix_t* dblock, const collage_matrix_t* dgate,
                                                    void* dpost_weight, void* dpre_weight, void* workspace, size_t workspace_bytes, void* stream) {
    return block_norm_backward(in, true, dy, dr, x, rstd_post, rstd_pre, dx, dblock, dgate, dpost_weight, dpre_weight, workspace, workspace_bytes, stream);
}

}  // extern "C"

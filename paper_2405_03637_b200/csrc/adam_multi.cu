// AdamW over many tensors in one launch, with states in 8 bits (codes with a scale for each 256 elements) or in floats; and the norm
// of all gradients.
//
//   m' = b1 m + c1 g,  v' = b2 v + c2 g^2,  x' = x - a (m' / bc1 / (sqrt(v' / bc2) + eps) + lam x)
//   8 bits: m = code * scale, sqrt(v) = code * scale; scales are the group's largest value / 448
//
// The root of v is kept rather than v: its 8 bits span 2^18, v would need twice that.  Its code is rounded with a random
// part, since in a step of beta2 = 0.999 it moves by a two-hundredth of a code's step, which rounding to nearest would undo each time;
// m moves by a tenth of what separates it from the gradient and is rounded to nearest.
// All of it is bound by memory: 10 (theta alone) to 16 bytes a parameter with 8-bit states, 22 to 28 with floats.
#include "adamw_float.cuh"
#include "ops_common.cuh"

#include <new>

namespace collage {
namespace ops {

constexpr uint32_t kGroup = 256;               // elements that share a scale: a warp's, eight a lane
constexpr uint32_t kAdamChunk = 4096;          // elements of a block's turn
constexpr int kAdamThreads = 256;

struct AdamRec {
    uint16_t* theta;
    void *rest, *m, *v;
    float *m_scale, *v_scale;
    const uint16_t* grad;
    uint64_t n, first;                         // first: position of its first element in the plan
    uint64_t aligned;                          // all arrays on 16 bytes (codes on 8)
};
struct AdamChunk {
    uint32_t tensor, index;
};

struct AdamScalars {
    Fp32Scalars f;
    float inv_bc1, inv_bc2, inv_root_bc2;      // 1 / bc1, 1 / bc2, 1 / sqrt(bc2)
    uint32_t key;
};

struct AdamArgs {
    const AdamRec* tensors;
    const AdamChunk* chunks;
    uint64_t num_chunks;
    const float* grad_scale;
    AdamScalars k;
};

__host__ __device__ __forceinline__ uint32_t mix32(uint32_t x) {
    x ^= x >> 16;
    x *= 0x6A09E667u;
    x ^= x >> 15;
    x *= 0xB504F333u;
    return x ^ (x >> 16);
}

__device__ __forceinline__ float fast_root(float x) {
    float r;
    asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// (theta, rest) + delta: the nearest bfloat16 to theta + RN(rest + delta), and what that lacks.  The sum is rounded to odd before it
// is rounded to bfloat16 (to nearest at once it would go astray at every tie of the float).
__device__ __forceinline__ void add_to_pair(float& theta, float& rest, float delta, uint32_t& theta_bits, uint32_t& rest_bits) {
    const float t = rest + delta, s = theta + t, back = s - theta;
    const float lost = (theta - (s - back)) + (t - back);                  // exact
    uint32_t bits = __float_as_uint(s);
    if (lost != 0.0f && fabsf(lost) < INFINITY) bits = (bits - ((__float_as_uint(lost) ^ bits) >> 31)) | 1u;
    theta_bits = to_bf16(__uint_as_float(bits));
    rest_bits = to_bf16((s - bf16_value(static_cast<uint16_t>(theta_bits))) + lost);
}

// What a lane holds of a group: values for eight elements, which ones those are is the caller's.
template <int STATE, int REST>
struct Octet {
    float g[8], theta[8], rest[8], m[8], v[8];           // STATE_E4M3: v is its root
    uint32_t theta_out[8], rest_out[8];                  // bits
};

template <int STATE, int REST>
__device__ __forceinline__ void update(Octet<STATE, REST>& o, const AdamScalars& k, float grad_scale) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float g = o.g[e] * grad_scale;
        const float x = REST == COLLAGE_REST_F32 ? o.rest[e] : REST == COLLAGE_REST_BF16 ? o.theta[e] + o.rest[e] : o.theta[e];
        float delta;
        if (STATE == COLLAGE_STATE_F32) {
            delta = adamw_fp32_delta(o.m[e], o.v[e], x, g, k.f);
        } else {
            const float m = __fmaf_rn(k.f.b1, o.m[e], k.f.c1 * g), v = __fmaf_rn(k.f.b2, o.v[e] * o.v[e], k.f.c2 * (g * g));
            const float root = fast_root(v);
            const float den = k.f.flags & COLLAGE_FLAG_EPS_INSIDE_SQRT ? fast_root(__fmaf_rn(v, k.inv_bc2, k.f.eps)) : __fmaf_rn(root, k.inv_root_bc2, k.f.eps);
            delta = k.f.neg_a * __fmaf_rn(k.f.lam, x, __fdividef(m * k.inv_bc1, den));
            o.m[e] = m;
            o.v[e] = root;
        }
        if (REST == COLLAGE_REST_BF16) {
            add_to_pair(o.theta[e], o.rest[e], delta, o.theta_out[e], o.rest_out[e]);
        } else {
            const float to = x + delta;
            o.rest[e] = to;
            o.theta_out[e] = to_bf16(to);
        }
    }
}

// Scale of a group from the bits of its largest absolute value, and what its values are taken times.
__device__ __forceinline__ float group_scale(uint32_t most, float& factor) {
    const float v = __uint_as_float(most);
    factor = v < 0x1p-100f ? 0.0f : most >= 0x7F800000u ? NAN : kE4m3Max / v;
    return v < 0x1p-100f ? 0.0f : most >= 0x7F800000u ? NAN : v * (1.0f / kE4m3Max);
}
// Code of a root before its last rounding, which is exact: rounded down after `random` (16 bits) of a step has been added.
// Below 2^-6 the codes are equally spaced, as they are from 2^-6 to 2^-5.
__device__ __forceinline__ float root_code(float root, float factor, uint32_t random) {
    const float u = root > 0.0f ? fmaxf(root * factor, 0x1p-9f) : 0.0f;
    const float shift = u < 0x1p-6f ? 0x1p-6f : 0.0f;
    return __uint_as_float((__float_as_uint(u + shift) + (random << 4)) & 0xFFF00000u) - shift;
}

__device__ __forceinline__ float2 e4m3_pair(uint32_t two) {
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(two), __NV_E4M3);
    return __half22float2(__half2(h));
}

// Eight consecutive floats
__device__ __forceinline__ void load8(const float* p, float (&f)[8]) {
    const float4 a = __ldcs(reinterpret_cast<const float4*>(p)), b = __ldcs(reinterpret_cast<const float4*>(p) + 1);
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
}
__device__ __forceinline__ void store8(float* p, const float (&f)[8]) {
    __stcs(reinterpret_cast<float4*>(p), make_float4(f[0], f[1], f[2], f[3]));
    __stcs(reinterpret_cast<float4*>(p) + 1, make_float4(f[4], f[5], f[6], f[7]));
}
__device__ __forceinline__ uint4 pack_words(const uint32_t (&b)[8]) {
    return make_uint4(b[0] | b[1] << 16, b[2] | b[3] << 16, b[4] | b[5] << 16, b[6] | b[7] << 16);
}

// One group of a tensor by a warp: whole and aligned, eight consecutive elements a lane.
template <int STATE, int REST>
__device__ __forceinline__ void whole_group(const AdamRec& t, uint64_t group, const AdamScalars& k, float grad_scale) {
    const int lane = threadIdx.x & 31;
    const uint64_t at = group * kGroup + lane * 8;
    Octet<STATE, REST> o;
    const uint4 qg = __ldcs(reinterpret_cast<const uint4*>(t.grad + at));
    uint4 qt = make_uint4(0, 0, 0, 0), qr = qt;
    uint2 qm = make_uint2(0, 0), qv = qm;
    float m_scale = 0.0f, v_scale = 0.0f;
    if (REST != COLLAGE_REST_F32) qt = __ldcs(reinterpret_cast<const uint4*>(t.theta + at));
    if (REST == COLLAGE_REST_BF16) qr = __ldcs(reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(t.rest) + at));
    if (REST == COLLAGE_REST_F32) load8(static_cast<const float*>(t.rest) + at, o.rest);
    if (STATE == COLLAGE_STATE_F32) {
        load8(static_cast<const float*>(t.m) + at, o.m);
        load8(static_cast<const float*>(t.v) + at, o.v);
    } else {
        qm = __ldcs(reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(t.m) + at));
        qv = __ldcs(reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(t.v) + at));
        m_scale = t.m_scale[group];
        v_scale = t.v_scale[group];
    }
    unpack8(qg, o.g);
    if (REST != COLLAGE_REST_F32) unpack8(qt, o.theta);
    if (REST == COLLAGE_REST_BF16) unpack8(qr, o.rest);
    if (STATE == COLLAGE_STATE_E4M3) {
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            const float2 m = e4m3_pair((e < 4 ? qm.x : qm.y) >> (8 * (e & 2))), v = e4m3_pair((e < 4 ? qv.x : qv.y) >> (8 * (e & 2)));
            o.m[e] = m.x * m_scale; o.m[e + 1] = m.y * m_scale;
            o.v[e] = v.x * v_scale; o.v[e + 1] = v.y * v_scale;
        }
    }
    update<STATE, REST>(o, k, grad_scale);
    __stcs(reinterpret_cast<uint4*>(t.theta + at), pack_words(o.theta_out));
    if (REST == COLLAGE_REST_BF16) __stcs(reinterpret_cast<uint4*>(static_cast<uint16_t*>(t.rest) + at), pack_words(o.rest_out));
    if (REST == COLLAGE_REST_F32) store8(static_cast<float*>(t.rest) + at, o.rest);
    if (STATE == COLLAGE_STATE_F32) {
        store8(static_cast<float*>(t.m) + at, o.m);
        store8(static_cast<float*>(t.v) + at, o.v);
        return;
    }
    uint32_t most_m = 0, most_v = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        most_m = max(most_m, __float_as_uint(o.m[e]) & 0x7FFFFFFFu);
        most_v = max(most_v, __float_as_uint(o.v[e]) & 0x7FFFFFFFu);
    }
    float m_factor, v_factor;
    m_scale = group_scale(__reduce_max_sync(0xFFFFFFFFu, most_m), m_factor);
    v_scale = group_scale(__reduce_max_sync(0xFFFFFFFFu, most_v), v_factor);
    const uint64_t pair = (t.first + at) >> 1;
    const uint32_t base = static_cast<uint32_t>(pair) + mix32(static_cast<uint32_t>(pair >> 32) + k.key);
    uint32_t wm[2] = {0, 0}, wv[2] = {0, 0};
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
        const uint32_t h = mix32(base + e / 2);                // (four pairs from a multiple of four on: no carry)
        wm[e >> 2] |= pack_e4m3(o.m[e] * m_factor, o.m[e + 1] * m_factor) << (8 * (e & 2));
        wv[e >> 2] |= pack_e4m3(root_code(o.v[e], v_factor, h & 0xFFFFu), root_code(o.v[e + 1], v_factor, h >> 16)) << (8 * (e & 2));
    }
    __stcs(reinterpret_cast<uint2*>(static_cast<uint8_t*>(t.m) + at), make_uint2(wm[0], wm[1]));
    __stcs(reinterpret_cast<uint2*>(static_cast<uint8_t*>(t.v) + at), make_uint2(wv[0], wv[1]));
    if (lane == 0) {
        t.m_scale[group] = m_scale;
        t.v_scale[group] = v_scale;
    }
}

// The same for groups that are cut short or not aligned: every 32nd element a lane.  Elements behind the end count as zeros.
template <int STATE, int REST>
__device__ __noinline__ void any_group(const AdamRec& t, uint64_t group, const AdamScalars& k, float grad_scale) {
    const int lane = threadIdx.x & 31;
    const uint64_t begin = group * kGroup;
    Octet<STATE, REST> o;
    float m_scale = 0.0f, v_scale = 0.0f;
    if (STATE == COLLAGE_STATE_E4M3) { m_scale = t.m_scale[group]; v_scale = t.v_scale[group]; }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint64_t i = begin + e * 32 + lane;
        o.g[e] = o.theta[e] = o.rest[e] = o.m[e] = o.v[e] = 0.0f;
        if (i >= t.n) continue;
        o.g[e] = bf16_value(t.grad[i]);
        if (REST != COLLAGE_REST_F32) o.theta[e] = bf16_value(t.theta[i]);
        if (REST == COLLAGE_REST_BF16) o.rest[e] = bf16_value(static_cast<const uint16_t*>(t.rest)[i]);
        if (REST == COLLAGE_REST_F32) o.rest[e] = static_cast<const float*>(t.rest)[i];
        if (STATE == COLLAGE_STATE_F32) {
            o.m[e] = static_cast<const float*>(t.m)[i];
            o.v[e] = static_cast<const float*>(t.v)[i];
        } else {
            o.m[e] = e4m3_pair(static_cast<const uint8_t*>(t.m)[i]).x * m_scale;
            o.v[e] = e4m3_pair(static_cast<const uint8_t*>(t.v)[i]).x * v_scale;
        }
    }
    update<STATE, REST>(o, k, grad_scale);
    uint32_t most_m = 0, most_v = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint64_t i = begin + e * 32 + lane;
        if (i >= t.n) continue;
        t.theta[i] = static_cast<uint16_t>(o.theta_out[e]);
        if (REST == COLLAGE_REST_BF16) static_cast<uint16_t*>(t.rest)[i] = static_cast<uint16_t>(o.rest_out[e]);
        if (REST == COLLAGE_REST_F32) static_cast<float*>(t.rest)[i] = o.rest[e];
        if (STATE == COLLAGE_STATE_F32) {
            static_cast<float*>(t.m)[i] = o.m[e];
            static_cast<float*>(t.v)[i] = o.v[e];
        }
        most_m = max(most_m, __float_as_uint(o.m[e]) & 0x7FFFFFFFu);
        most_v = max(most_v, __float_as_uint(o.v[e]) & 0x7FFFFFFFu);
    }
    if (STATE == COLLAGE_STATE_F32) return;
    float m_factor, v_factor;
    m_scale = group_scale(__reduce_max_sync(0xFFFFFFFFu, most_m), m_factor);
    v_scale = group_scale(__reduce_max_sync(0xFFFFFFFFu, most_v), v_factor);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint64_t i = begin + e * 32 + lane;
        if (i >= t.n) continue;
        const uint64_t pair = (t.first + i) >> 1;
        const uint32_t h = mix32(static_cast<uint32_t>(pair) + mix32(static_cast<uint32_t>(pair >> 32) + k.key));
        static_cast<uint8_t*>(t.m)[i] = to_e4m3(o.m[e] * m_factor);
        static_cast<uint8_t*>(t.v)[i] = to_e4m3(root_code(o.v[e], v_factor, i & 1 ? h >> 16 : h & 0xFFFFu));
    }
    if (lane == 0) {
        t.m_scale[group] = m_scale;
        t.v_scale[group] = v_scale;
    }
}

template <int STATE, int REST>
__global__ void __launch_bounds__(kAdamThreads) adam_step_kernel(const __grid_constant__ AdamArgs a) {
    after_previous();
    const float grad_scale = a.grad_scale ? *a.grad_scale : 1.0f;
    for (uint64_t c = blockIdx.x; c < a.num_chunks; c += gridDim.x) {
        const AdamChunk chunk = a.chunks[c];
        const AdamRec& t = a.tensors[chunk.tensor];
        const uint64_t first = chunk.index * static_cast<uint64_t>(kAdamChunk / kGroup), end = (t.n + kGroup - 1) / kGroup;
        const bool aligned = t.aligned;
        for (uint64_t g = first + (threadIdx.x >> 5); g < min(first + kAdamChunk / kGroup, end); g += kAdamThreads / 32) {
            if (aligned && (g + 1) * kGroup <= t.n)
                whole_group<STATE, REST>(t, g, a.k, grad_scale);
            else
                any_group<STATE, REST>(t, g, a.k, grad_scale);
        }
    }
}

// ---------------------------------------------------------------------------------------------------------- norm ---

struct NormArgs {
    const AdamRec* tensors;
    const AdamChunk* chunks;
    uint64_t num_chunks;
    EdqPartial* partials;
    unsigned int* ticket;
    float *norm, *grad_scale;
    double max_norm;
};

// Sum of squares of eight values: in floats where no square and no digit is lost, else in 64 bits.
__device__ __forceinline__ double squares(const float (&g)[8]) {
    float sum = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) sum = __fmaf_rn(g[e], g[e], sum);
    if (sum > 0x1p-100f && sum < 0x1p120f) return sum;
    double exact = 0.0;
#pragma unroll
    for (int e = 0; e < 8; ++e) exact = __fma_rn(static_cast<double>(g[e]), static_cast<double>(g[e]), exact);
    return exact;
}

__global__ void __launch_bounds__(kAdamThreads) grad_norm_kernel(const __grid_constant__ NormArgs a) {
    __shared__ double part[kAdamThreads / 32];
    __shared__ bool is_last;
    after_previous();
    double sum = 0.0;
    for (uint64_t c = blockIdx.x; c < a.num_chunks; c += gridDim.x) {
        const AdamChunk chunk = a.chunks[c];
        const AdamRec& t = a.tensors[chunk.tensor];
        const uint64_t begin = chunk.index * static_cast<uint64_t>(kAdamChunk);
        float g[2][8];
        if (t.aligned && begin + kAdamChunk <= t.n) {
            const uint4* q = reinterpret_cast<const uint4*>(t.grad + begin) + threadIdx.x;
            unpack8(q[0], g[0]);
            unpack8(q[kAdamThreads], g[1]);
        } else {
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint64_t j = begin + (i * 8 + e) * kAdamThreads + threadIdx.x;
                    g[i][e] = j < t.n ? bf16_value(t.grad[j]) : 0.0f;
                }
        }
        sum += squares(g[0]);
        sum += squares(g[1]);
    }
    auto joined = [&](double v) {              // over the block, in a fixed order; the result in the first warp
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
        __syncthreads();
        if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
        __syncthreads();
        v = (threadIdx.x & 31) < kAdamThreads / 32 ? part[threadIdx.x & 31] : 0.0;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
        return v;
    };
    sum = joined(sum);
    // the block that draws the last ticket adds the blocks' sums up; nobody waits
    if (threadIdx.x == 0) {
        a.partials[blockIdx.x].sq = sum;
        __threadfence();
        const unsigned int last = gridDim.x - 1;
        unsigned int drawn = atomicInc(a.ticket, last);
        if (drawn > last) drawn = atomicInc(a.ticket, last);           // (never a count: the word was not zeroed)
        is_last = drawn == last;
    }
    __syncthreads();
    if (!is_last) return;
    __threadfence();
    sum = 0.0;
    for (unsigned int i = threadIdx.x; i < gridDim.x; i += kAdamThreads) sum += __ldcg(&a.partials[i].sq);
    sum = joined(sum);
    if (threadIdx.x == 0) {
        const double norm = sqrt(sum);
        *a.norm = static_cast<float>(norm);
        if (a.grad_scale) *a.grad_scale = norm > a.max_norm ? static_cast<float>(a.max_norm / norm) : norm == norm ? 1.0f : NAN;
    }
}

}  // namespace ops
}  // namespace collage

using namespace collage;
using namespace collage::ops;

struct collage_adam_plan {
    AdamRec* d_tensors = nullptr;
    AdamChunk* d_chunks = nullptr;
    uint64_t num_chunks = 0;
    std::vector<ByteRange> ranges, written;    // sorted by address: all arrays, and those that a step writes
    int state = 0, rest = 0, device = -1;
    ~collage_adam_plan() {
        cudaFree(d_tensors);
        cudaFree(d_chunks);
    }
};

namespace {

collage_status_t create(const collage_adam_tensor_t* tensors, int num, int state, int rest, collage_adam_plan** out) {
    const uint64_t state_bytes = state == COLLAGE_STATE_F32 ? 4 : 1, rest_bytes = rest == COLLAGE_REST_F32 ? 4 : 2;
    std::vector<ByteRange> ranges, written;
    std::vector<AdamRec> recs;
    std::vector<AdamChunk> chunks;
    uint64_t first = 0, num_chunks = 0;
    for (int i = 0; i < num; ++i) {
        const collage_adam_tensor_t& t = tensors[i];
        if (t.n > (1ull << 58)) return COLLAGE_ERR_ARG;
        if (t.n == 0) continue;
        const bool codes = state == COLLAGE_STATE_E4M3;
        if ((!codes && (t.m_scale || t.v_scale)) || (rest == COLLAGE_REST_NONE && t.rest)) return COLLAGE_ERR_ARG;
        if (!t.theta || !t.m || !t.v || !t.grad || (rest != COLLAGE_REST_NONE && !t.rest) || (codes && (!t.m_scale || !t.v_scale))) return COLLAGE_ERR_NULL;
        auto off = [](const void* p, uint64_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes != 0; };
        if (off(t.theta, 2) || off(t.grad, 2) || off(t.rest, rest_bytes) || off(t.m, state_bytes) || off(t.v, state_bytes) || off(t.m_scale, 4) || off(t.v_scale, 4))
            return COLLAGE_ERR_ARG;
        const uint64_t groups = (t.n + kGroup - 1) / kGroup, own_chunks = (t.n + kAdamChunk - 1) / kAdamChunk;
        num_chunks += own_chunks;
        if (num_chunks > 0xFFFFFFFFull) return COLLAGE_ERR_ARG;
        push_bytes(ranges, t.grad, 2 * t.n);
        auto out_array = [&](const void* p, uint64_t bytes) {
            push_bytes(ranges, p, bytes);
            push_bytes(written, p, bytes);
        };
        out_array(t.theta, 2 * t.n);
        out_array(t.rest, rest_bytes * t.n);
        out_array(t.m, state_bytes * t.n);
        out_array(t.v, state_bytes * t.n);
        out_array(t.m_scale, 4 * groups);
        out_array(t.v_scale, 4 * groups);
        AdamRec r = {};
        r.theta = static_cast<uint16_t*>(t.theta);
        r.rest = t.rest;
        r.m = t.m;
        r.v = t.v;
        r.m_scale = t.m_scale;
        r.v_scale = t.v_scale;
        r.grad = static_cast<const uint16_t*>(t.grad);
        r.n = t.n;
        r.first = first;
        r.aligned = !off(t.theta, 16) && !off(t.grad, 16) && !off(t.rest, 16) && !off(t.m, codes ? 8 : 16) && !off(t.v, codes ? 8 : 16);
        first += groups * kGroup;
        for (uint64_t c = 0; c < own_chunks; ++c) chunks.push_back({static_cast<uint32_t>(recs.size()), static_cast<uint32_t>(c)});
        recs.push_back(r);
    }
    if (any_overlap(ranges)) return COLLAGE_ERR_ALIAS;
    any_overlap(written);                      // (sorts)
    DeviceInfo dev;
    if (const collage_status_t st = current_device(&dev); st != COLLAGE_OK) return st;
    collage_adam_plan* plan = new collage_adam_plan;
    plan->num_chunks = num_chunks;
    plan->ranges = std::move(ranges);
    plan->written = std::move(written);
    plan->state = state;
    plan->rest = rest;
    if (cudaGetDevice(&plan->device) != cudaSuccess ||
        (num_chunks && (cudaMalloc(&plan->d_tensors, recs.size() * sizeof(AdamRec)) != cudaSuccess ||
                        cudaMalloc(&plan->d_chunks, chunks.size() * sizeof(AdamChunk)) != cudaSuccess ||
                        cudaMemcpy(plan->d_tensors, recs.data(), recs.size() * sizeof(AdamRec), cudaMemcpyHostToDevice) != cudaSuccess ||
                        cudaMemcpy(plan->d_chunks, chunks.data(), chunks.size() * sizeof(AdamChunk), cudaMemcpyHostToDevice) != cudaSuccess))) {
        delete plan;
        return COLLAGE_ERR_CUDA;
    }
    *out = plan;
    return COLLAGE_OK;
}

bool on_its_device(const collage_adam_plan* plan) {
    int device = -1;
    return cudaGetDevice(&device) == cudaSuccess && device == plan->device;
}

}  // namespace

extern "C" {

collage_status_t collage_adam_plan_create(const collage_adam_tensor_t* tensors, int num, collage_adam_state_t state, collage_adam_rest_t rest,
                                          collage_adam_plan_t** out_plan) {
    if (!out_plan) return COLLAGE_ERR_NULL;
    *out_plan = nullptr;
    if (num < 0 || (state != COLLAGE_STATE_F32 && state != COLLAGE_STATE_E4M3) || rest < COLLAGE_REST_NONE || rest > COLLAGE_REST_F32) return COLLAGE_ERR_ARG;
    if (!tensors && num) return COLLAGE_ERR_NULL;
    try {
        return create(tensors, num, state, rest, out_plan);
    } catch (const std::bad_alloc&) {
        return COLLAGE_ERR_LIMIT;
    }
}

collage_status_t collage_adam_plan_destroy(collage_adam_plan_t* plan) {
    delete plan;
    return COLLAGE_OK;
}

collage_status_t collage_adam_step(const collage_adam_plan_t* plan, const collage_hyper_t* hyper, uint64_t step, uint64_t seed, const float* grad_scale,
                                   void* stream) {
    if (!plan || !hyper) return COLLAGE_ERR_NULL;
    if (step == 0 || !hyper_in_range(hyper) || hyper->edq_out || reinterpret_cast<uintptr_t>(grad_scale) % 4) return COLLAGE_ERR_ARG;
    if (hyper->flags & ~(COLLAGE_FLAG_EPS_INSIDE_SQRT | COLLAGE_FLAG_PIPELINE_KERNEL | COLLAGE_FLAG_DIRECT_KERNEL | COLLAGE_FLAG_LARGE_TILES))
        return COLLAGE_ERR_ARG;
    if (overlaps_sorted(plan->written, grad_scale, 4)) return COLLAGE_ERR_ALIAS;
    DeviceInfo dev;
    if (const collage_status_t st = current_device(&dev); st != COLLAGE_OK) return st;
    if (!on_its_device(plan)) return COLLAGE_ERR_ARG;
    if (plan->num_chunks == 0) return COLLAGE_OK;
    AdamArgs a = {};
    a.tensors = plan->d_tensors;
    a.chunks = plan->d_chunks;
    a.num_chunks = plan->num_chunks;
    a.grad_scale = grad_scale;
    a.k.f = fp32_scalars(hyper, step);
    const double t = static_cast<double>(step), bc1 = 1.0 - std::pow(hyper->beta1, t), bc2 = 1.0 - std::pow(hyper->beta2, t);
    a.k.inv_bc1 = static_cast<float>(1.0 / bc1);
    a.k.inv_bc2 = static_cast<float>(1.0 / bc2);
    a.k.inv_root_bc2 = static_cast<float>(1.0 / std::sqrt(bc2));
    uint32_t key = mix32(static_cast<uint32_t>(step >> 32));
    for (const uint64_t word : {step, seed >> 32, seed}) key = mix32(static_cast<uint32_t>(word) + key);
    a.k.key = key;
    const uint64_t grid = std::min<uint64_t>(plan->num_chunks, (1ull << 31) - 1);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    switch (plan->state * 3 + plan->rest) {
        case 0: return launch<&adam_step_kernel<0, 0>>(grid, kAdamThreads, 1, 0, s, a);
        case 1: return launch<&adam_step_kernel<0, 1>>(grid, kAdamThreads, 1, 0, s, a);
        case 2: return launch<&adam_step_kernel<0, 2>>(grid, kAdamThreads, 1, 0, s, a);
        case 3: return launch<&adam_step_kernel<1, 0>>(grid, kAdamThreads, 1, 0, s, a);
        case 4: return launch<&adam_step_kernel<1, 1>>(grid, kAdamThreads, 1, 0, s, a);
        default: return launch<&adam_step_kernel<1, 2>>(grid, kAdamThreads, 1, 0, s, a);
    }
}

collage_status_t collage_adam_grad_norm(const collage_adam_plan_t* plan, double max_norm, float* norm, float* grad_scale, void* workspace,
                                        size_t workspace_bytes, void* stream) {
    if (!plan || !norm) return COLLAGE_ERR_NULL;
    if (!(max_norm > 0.0) || reinterpret_cast<uintptr_t>(norm) % 4 || reinterpret_cast<uintptr_t>(grad_scale) % 4) return COLLAGE_ERR_ARG;
    if (!workspace || workspace_bytes < kWorkspaceBytes || reinterpret_cast<uintptr_t>(workspace) % 16) return COLLAGE_ERR_WORKSPACE;
    AliasCheck alias;
    alias.add(span_of(norm, 4), true);
    alias.add(span_of(grad_scale, grad_scale ? 4 : 0), true);
    alias.add(span_of(workspace, kWorkspaceBytes), true);
    if (alias.clash() || overlaps_sorted(plan->ranges, norm, 4) || overlaps_sorted(plan->ranges, grad_scale, 4) ||
        overlaps_sorted(plan->ranges, workspace, kWorkspaceBytes))
        return COLLAGE_ERR_ALIAS;
    DeviceInfo dev;
    if (const collage_status_t st = current_device(&dev); st != COLLAGE_OK) return st;
    if (!on_its_device(plan)) return COLLAGE_ERR_ARG;
    NormArgs a = {};
    a.tensors = plan->d_tensors;
    a.chunks = plan->d_chunks;
    a.num_chunks = plan->num_chunks;
    a.partials = static_cast<EdqPartial*>(workspace);
    a.ticket = reinterpret_cast<unsigned int*>(static_cast<char*>(workspace) + kTicketOffset);
    a.norm = norm;
    a.grad_scale = grad_scale;
    a.max_norm = max_norm;
    const uint64_t grid = std::max<uint64_t>(1, std::min<uint64_t>({plan->num_chunks, 8ull * dev.sm_count, static_cast<uint64_t>(kMaxGrid)}));
    return launch<&grad_norm_kernel>(grid, kAdamThreads, 1, 0, static_cast<cudaStream_t>(stream), a);
}

}  // extern "C"

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
constexpr uint32_t kAdamChunk = 4096;          // elements of the norm's turns
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
    const AdamChunk* tasks;                    // task: task_groups groups of a tensor, for one warp
    uint64_t num_tasks;
    uint32_t task_groups;
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

__device__ __forceinline__ uint64_t pair_of(float v) { return ops::pair_of(v, v); }
__device__ __forceinline__ uint64_t sub_pair(uint64_t a, uint64_t b) { return fma_pair(b, pair_of(-1.0f), a); }
__device__ __forceinline__ uint64_t bf16_pair(uint32_t word) { return ops::pair_of(bf16_lo(word), bf16_hi(word)); }
__device__ __forceinline__ uint64_t e4m3_pair(uint32_t two) {
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(two), __NV_E4M3);
    const float2 f = __half22float2(__half2(h));
    return ops::pair_of(f.x, f.y);
}

// Square roots: y = rsqrt(v) gives r = v y, and a step of Newton's method on r^2 = v, whose remainder r^2 - v is exact in an fma, the
// correctly rounded root but for a few in a million (in half the instructions of one that always is).
__device__ __forceinline__ uint64_t root_pair(uint64_t v) {
    const float2 f = floats_of(v);
    float2 y;
    asm("rsqrt.approx.f32 %0, %1;" : "=f"(y.x) : "f"(fmaxf(f.x, 0x1p-149f)));         // (of 0: 0 times a finite number)
    asm("rsqrt.approx.f32 %0, %1;" : "=f"(y.y) : "f"(fmaxf(f.y, 0x1p-149f)));
    const uint64_t y2 = ops::pair_of(y.x, y.y), r = mul_pair(v, y2);
    return fma_pair(fma_pair(r, r, mul_pair(v, pair_of(-1.0f))), mul_pair(y2, pair_of(-0.5f)), r);
}
__device__ __forceinline__ uint64_t reciprocal_pair(uint64_t v) {
    float2 f = floats_of(v);
    asm("rcp.approx.f32 %0, %0;" : "+f"(f.x));
    asm("rcp.approx.f32 %0, %0;" : "+f"(f.y));
    return ops::pair_of(f.x, f.y);
}

// (theta, rest) + delta: theta' is the bfloat16 nearest to theta + RN(rest + delta), rest' what that lacks.
__device__ __forceinline__ void add_to_pair(uint64_t theta, uint64_t rest, uint64_t delta, uint32_t& theta_word, uint32_t& rest_word) {
    const uint64_t t = add_pair(rest, delta), s = add_pair(theta, t), back = sub_pair(s, theta);
    const uint64_t lost = add_pair(sub_pair(theta, sub_pair(s, back)), sub_pair(t, back));                  // exact: theta + t = s + lost
    const float2 sum = floats_of(s);
    theta_word = pack_bf16(sum.x, sum.y);
    // A float half-way between two bfloat16 values: which one is nearer hangs on what the float has lost.  It is rounded to odd first,
    // towards the sum's own side.  (One in 65536; the test finds a half-word of 0x8000, and now and then another.)
    const uint32_t low = __byte_perm(__float_as_uint(sum.x), __float_as_uint(sum.y), 0x5410) ^ 0x80008000u;
    if ((low - 0x00010001u) & ~low & 0x80008000u) {
        const float2 l = floats_of(lost);
        auto odd = [](float f, float rest_of) {
            const uint32_t bits = __float_as_uint(f);
            const bool off = rest_of != 0.0f && fabsf(rest_of) < INFINITY;
            return __uint_as_float(off ? (bits - ((__float_as_uint(rest_of) ^ bits) >> 31)) | 1u : bits);
        };
        theta_word = pack_bf16(odd(sum.x, l.x), odd(sum.y, l.y));
    }
    const float2 r = floats_of(add_pair(sub_pair(s, bf16_pair(theta_word)), lost));
    rest_word = pack_bf16(r.x, r.y);
}

// Eight elements of a lane, in pairs, before and behind the update.  With states in 8 bits v is its root.
struct Octet {
    uint64_t g[4], theta[4], rest[4], m[4], v[4];
    uint32_t theta_out[4], rest_out[4];                  // two bfloat16 each
};

template <int STATE, int REST>
__device__ __forceinline__ void update(Octet& o, const AdamScalars& k, float grad_scale) {
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const uint64_t g = mul_pair(o.g[p], pair_of(grad_scale));
        const uint64_t x = REST == COLLAGE_REST_F32 ? o.rest[p] : REST == COLLAGE_REST_BF16 ? add_pair(o.theta[p], o.rest[p]) : o.theta[p];
        uint64_t delta;
        if (STATE == COLLAGE_STATE_F32) {
            float2 m = floats_of(o.m[p]), v = floats_of(o.v[p]);
            const float2 gf = floats_of(g), xf = floats_of(x);
            const float lo = adamw_fp32_delta(m.x, v.x, xf.x, gf.x, k.f), hi = adamw_fp32_delta(m.y, v.y, xf.y, gf.y, k.f);
            delta = ops::pair_of(lo, hi);
            o.m[p] = ops::pair_of(m.x, m.y);
            o.v[p] = ops::pair_of(v.x, v.y);
        } else {
            // every product and sum of the states is rounded once, so that their codes hang on nothing but the formulas
            const uint64_t m = add_pair(mul_pair(o.m[p], pair_of(k.f.b1)), mul_pair(g, pair_of(k.f.c1)));
            const uint64_t v = add_pair(mul_pair(mul_pair(o.v[p], o.v[p]), pair_of(k.f.b2)), mul_pair(mul_pair(g, g), pair_of(k.f.c2)));
            const uint64_t root = root_pair(v);
            uint64_t den;
            if (k.f.flags & COLLAGE_FLAG_EPS_INSIDE_SQRT)
                den = root_pair(fma_pair(v, pair_of(k.inv_bc2), pair_of(k.f.eps)));
            else
                den = fma_pair(root, pair_of(k.inv_root_bc2), pair_of(k.f.eps));
            const uint64_t part = mul_pair(mul_pair(m, pair_of(k.inv_bc1)), reciprocal_pair(den));
            delta = mul_pair(fma_pair(x, pair_of(k.f.lam), part), pair_of(k.f.neg_a));
            o.m[p] = m;
            o.v[p] = root;
        }
        if (REST == COLLAGE_REST_BF16) {
            add_to_pair(o.theta[p], o.rest[p], delta, o.theta_out[p], o.rest_out[p]);
        } else {
            o.rest[p] = add_pair(x, delta);
            const float2 to = floats_of(o.rest[p]);
            o.theta_out[p] = pack_bf16(to.x, to.y);
        }
    }
}

// Largest absolute value of eight over the warp; NaN where there is one.
__device__ __forceinline__ uint32_t largest(const uint64_t (&f)[4]) {
    float most = 0.0f;
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const float2 v = floats_of(f[p]);
        asm("max.NaN.f32 %0, %0, %1;" : "+f"(most) : "f"(fabsf(v.x)));
        asm("max.NaN.f32 %0, %0, %1;" : "+f"(most) : "f"(fabsf(v.y)));
    }
    return __reduce_max_sync(0xFFFFFFFFu, __float_as_uint(most));
}
// Scale of a group from the bits of its largest absolute value, and what its values are taken times.
__device__ __forceinline__ float group_scale(uint32_t most, float& factor) {
    const float v = __uint_as_float(most);
    factor = v < 0x1p-100f ? 0.0f : most >= 0x7F800000u ? NAN : 1.0f / v * kE4m3Max;
    return v < 0x1p-100f ? 0.0f : most >= 0x7F800000u ? NAN : v * (1.0f / kE4m3Max);
}
// Codes of values to nearest even, as bytes.
__device__ __forceinline__ uint2 nearest_codes(const uint64_t (&f)[4], float factor) {
    uint32_t w[4];
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const float2 v = floats_of(mul_pair(f[p], pair_of(factor)));
        w[p] = pack_e4m3(v.x, v.y);
    }
    return make_uint2(__byte_perm(w[0], w[1], 0x5410), __byte_perm(w[2], w[3], 0x5410));
}
// Codes of roots, rounded down after `random` (16 bits for each; two in a word) of a step has been added.  From 2^-6 on a code is the
// upper bits of the float, less the difference of the exponents' biases; below, codes are equally spaced, as they are from 2^-6 to 2^-5.
__device__ __forceinline__ uint2 random_codes(const uint64_t (&f)[4], float factor, const uint32_t (&random)[4]) {
    float u[8], least = INFINITY;
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const float2 v = floats_of(mul_pair(f[p], pair_of(factor)));
        u[2 * p] = v.x;
        u[2 * p + 1] = v.y;
        least = fminf(least, fminf(v.x, v.y));
    }
    uint32_t code[8];
    if (least >= 0x1p-6f) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {              // random << 8 below, 0x40 above: (127 - 7) << 27 less, modulo 2^32
            const uint32_t r = __byte_perm(random[e / 2], 0x40u, e & 1 ? 0x4325 : 0x4105);
            code[e] = (__float_as_uint(u[e]) << 4) + r;
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float2 root = floats_of(f[e / 2]);
            const float v = (e & 1 ? root.y : root.x) > 0.0f ? fmaxf(u[e], 0x1p-9f) : 0.0f, shift = v < 0x1p-6f ? 0x1p-6f : 0.0f;
            const uint32_t part = e & 1 ? random[e / 2] >> 16 : random[e / 2] & 0xFFFFu;
            code[e] = static_cast<uint32_t>(to_e4m3(__uint_as_float((__float_as_uint(v + shift) + (part << 4)) & 0xFFF00000u) - shift)) << 24;
        }
    }
    uint32_t w[4];
#pragma unroll
    for (int p = 0; p < 4; ++p) w[p] = __byte_perm(code[2 * p], code[2 * p + 1], 0x7373);
    return make_uint2(__byte_perm(w[0], w[1], 0x5410), __byte_perm(w[2], w[3], 0x5410));
}
__device__ __forceinline__ uint32_t random_word(uint64_t pair, uint32_t key) {
    return mix32(static_cast<uint32_t>(pair) + mix32(static_cast<uint32_t>(pair >> 32) + key));
}

// Which elements of a whole group a lane has: eight in a row, or, where some array is of floats, four in a row of each half, so that
// every access of a warp is to consecutive bytes.  A lane's bytes of a group of each array in shared memory, `kStages` groups ahead.
template <int STATE, int REST>
struct Form {
    static constexpr bool kHalves = STATE == COLLAGE_STATE_F32 || REST == COLLAGE_REST_F32;
    static constexpr bool kTheta = REST != COLLAGE_REST_F32;
    static constexpr uint32_t kStateBytes = STATE == COLLAGE_STATE_F32 ? 4 : 1, kRestBytes = REST == COLLAGE_REST_F32 ? 4 : REST == COLLAGE_REST_BF16 ? 2 : 0;
    // offsets of the arrays in a stage
    static constexpr uint32_t kG = 0, kT = kG + 2 * kGroup, kR = kT + (kTheta ? 2 * kGroup : 0), kM = kR + kRestBytes * kGroup, kV = kM + kStateBytes * kGroup,
                              kScales = kV + kStateBytes * kGroup, kStage = kScales + 16;
    static constexpr int kStages = 3;
    static __device__ __forceinline__ uint32_t element(int lane, int half) { return kHalves ? half * (kGroup / 2) + lane * 4 : lane * 8 + half * 4; }
};
constexpr int kAdamWarps = kAdamThreads / 32;

template <uint32_t BYTES>
__device__ __forceinline__ void copy_async(uint32_t to, const void* from) {
    if constexpr (BYTES == 16)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
    else
        asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(to), "l"(from), "n"(BYTES) : "memory");
}

// Sends for a lane's part of one array of a whole group, which begins at `from`.
template <typename F, uint32_t BYTES>
__device__ __forceinline__ void send_array(uint32_t stage, const void* from, int lane) {
    const char* p = static_cast<const char*>(from);
    if constexpr (F::kHalves) {
#pragma unroll
        for (int h = 0; h < 2; ++h) copy_async<4 * BYTES>(stage + F::element(lane, h) * BYTES, p + F::element(lane, h) * BYTES);
    } else {
        copy_async<8 * BYTES>(stage + lane * 8 * BYTES, p + lane * 8 * BYTES);
    }
}
// Its eight elements, in 16, 32 or 64 bytes of words
template <typename F, uint32_t BYTES>
__device__ __forceinline__ void fetch_array(const uint8_t* stage, int lane, uint32_t (&w)[2 * BYTES]) {
    constexpr int kHalf = BYTES;               // words of four elements
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t* p = reinterpret_cast<const uint32_t*>(stage + F::element(lane, h) * BYTES);
        if constexpr (kHalf == 4) {
            const uint4 q = *reinterpret_cast<const uint4*>(p);
            w[h * 4] = q.x; w[h * 4 + 1] = q.y; w[h * 4 + 2] = q.z; w[h * 4 + 3] = q.w;
        } else if constexpr (kHalf == 2) {
            const uint2 q = *reinterpret_cast<const uint2*>(p);
            w[h * 2] = q.x; w[h * 2 + 1] = q.y;
        } else {
            w[h] = *p;
        }
    }
}
template <typename F, uint32_t BYTES>
__device__ __forceinline__ void store_array(void* to, int lane, const uint32_t (&w)[2 * BYTES]) {
    char* p = static_cast<char*>(to);
    if constexpr (!F::kHalves && BYTES == 2) {
        __stcs(reinterpret_cast<uint4*>(p + lane * 16), make_uint4(w[0], w[1], w[2], w[3]));
    } else if constexpr (!F::kHalves && BYTES == 1) {
        __stcs(reinterpret_cast<uint2*>(p + lane * 8), make_uint2(w[0], w[1]));
    } else {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            char* q = p + F::element(lane, h) * BYTES;
            if constexpr (BYTES == 4) __stcs(reinterpret_cast<uint4*>(q), make_uint4(w[4 * h], w[4 * h + 1], w[4 * h + 2], w[4 * h + 3]));
            if constexpr (BYTES == 2) __stcs(reinterpret_cast<uint2*>(q), make_uint2(w[2 * h], w[2 * h + 1]));
            if constexpr (BYTES == 1) __stcs(reinterpret_cast<uint32_t*>(q), w[h]);
        }
    }
}
__device__ __forceinline__ void floats_to_words(const uint64_t (&f)[4], uint32_t (&w)[8]) {
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const float2 v = floats_of(f[p]);
        w[2 * p] = __float_as_uint(v.x);
        w[2 * p + 1] = __float_as_uint(v.y);
    }
}
__device__ __forceinline__ void words_to_floats(const uint32_t (&w)[8], uint64_t (&f)[4]) {
#pragma unroll
    for (int p = 0; p < 4; ++p) f[p] = ops::pair_of(__uint_as_float(w[2 * p]), __uint_as_float(w[2 * p + 1]));
}

template <int STATE, int REST>
__device__ __forceinline__ void send_group(const AdamRec& t, uint64_t group, uint32_t stage, int lane) {
    using F = Form<STATE, REST>;
    const uint64_t at = group * kGroup;
    send_array<F, 2>(stage + F::kG, t.grad + at, lane);
    if constexpr (F::kTheta) send_array<F, 2>(stage + F::kT, t.theta + at, lane);
    if constexpr (F::kRestBytes) send_array<F, F::kRestBytes>(stage + F::kR, static_cast<const char*>(t.rest) + at * F::kRestBytes, lane);
    send_array<F, F::kStateBytes>(stage + F::kM, static_cast<const char*>(t.m) + at * F::kStateBytes, lane);
    send_array<F, F::kStateBytes>(stage + F::kV, static_cast<const char*>(t.v) + at * F::kStateBytes, lane);
    if (STATE == COLLAGE_STATE_E4M3 && lane < 2) copy_async<4>(stage + F::kScales + 4 * lane, (lane ? t.v_scale : t.m_scale) + group);
}

// One group of a tensor by a warp: whole and aligned, its bytes in shared memory.
template <int STATE, int REST>
__device__ __forceinline__ void whole_group(const AdamRec& t, uint64_t group, const uint8_t* stage, const AdamScalars& k, float grad_scale, int lane) {
    using F = Form<STATE, REST>;
    const uint64_t at = group * kGroup;
    Octet o;
    uint32_t w[4];
    fetch_array<F, 2>(stage + F::kG, lane, w);
#pragma unroll
    for (int p = 0; p < 4; ++p) o.g[p] = bf16_pair(w[p]);
    if constexpr (F::kTheta) {
        fetch_array<F, 2>(stage + F::kT, lane, w);
#pragma unroll
        for (int p = 0; p < 4; ++p) o.theta[p] = bf16_pair(w[p]);
    }
    if constexpr (REST == COLLAGE_REST_BF16) {
        fetch_array<F, 2>(stage + F::kR, lane, w);
#pragma unroll
        for (int p = 0; p < 4; ++p) o.rest[p] = bf16_pair(w[p]);
    }
    uint32_t wide[8];
    if constexpr (REST == COLLAGE_REST_F32) {
        fetch_array<F, 4>(stage + F::kR, lane, wide);
        words_to_floats(wide, o.rest);
    }
    if constexpr (STATE == COLLAGE_STATE_F32) {
        fetch_array<F, 4>(stage + F::kM, lane, wide);
        words_to_floats(wide, o.m);
        fetch_array<F, 4>(stage + F::kV, lane, wide);
        words_to_floats(wide, o.v);
    } else {
        const float2 scales = *reinterpret_cast<const float2*>(stage + F::kScales);
        uint32_t c[2];
        fetch_array<F, 1>(stage + F::kM, lane, c);
#pragma unroll
        for (int p = 0; p < 4; ++p) o.m[p] = mul_pair(e4m3_pair(c[p / 2] >> (16 * (p & 1))), pair_of(scales.x));
        fetch_array<F, 1>(stage + F::kV, lane, c);
#pragma unroll
        for (int p = 0; p < 4; ++p) o.v[p] = mul_pair(e4m3_pair(c[p / 2] >> (16 * (p & 1))), pair_of(scales.y));
    }
    update<STATE, REST>(o, k, grad_scale);
    store_array<F, 2>(t.theta + at, lane, o.theta_out);
    if constexpr (REST == COLLAGE_REST_BF16) store_array<F, 2>(static_cast<uint16_t*>(t.rest) + at, lane, o.rest_out);
    if constexpr (REST == COLLAGE_REST_F32) {
        floats_to_words(o.rest, wide);
        store_array<F, 4>(static_cast<float*>(t.rest) + at, lane, wide);
    }
    if constexpr (STATE == COLLAGE_STATE_F32) {
        floats_to_words(o.m, wide);
        store_array<F, 4>(static_cast<float*>(t.m) + at, lane, wide);
        floats_to_words(o.v, wide);
        store_array<F, 4>(static_cast<float*>(t.v) + at, lane, wide);
    } else {
        float m_factor, v_factor;
        const float m_scale = group_scale(largest(o.m), m_factor), v_scale = group_scale(largest(o.v), v_factor);
        // the group's pairs begin at a multiple of 128, so their upper word is one
        const uint64_t pair = (t.first + at) >> 1;
        const uint32_t base = static_cast<uint32_t>(pair) + mix32(static_cast<uint32_t>(pair >> 32) + k.key);
        uint32_t random[4];
#pragma unroll
        for (int p = 0; p < 4; ++p) random[p] = mix32(base + F::element(lane, p / 2) / 2 + (p & 1));
        const uint2 cm = nearest_codes(o.m, m_factor), cv = random_codes(o.v, v_factor, random);
        const uint32_t wm[2] = {cm.x, cm.y}, wv[2] = {cv.x, cv.y};
        store_array<F, 1>(static_cast<uint8_t*>(t.m) + at, lane, wm);
        store_array<F, 1>(static_cast<uint8_t*>(t.v) + at, lane, wv);
        if (lane < 2) (lane ? t.v_scale : t.m_scale)[group] = lane ? v_scale : m_scale;
    }
}

// The same for groups that are cut short or not aligned: every 32nd element a lane.  Elements behind the end count as zeros.
template <int STATE, int REST>
__device__ __noinline__ void any_group(const AdamRec& t, uint64_t group, const AdamScalars& k, float grad_scale) {
    const int lane = threadIdx.x & 31;
    const uint64_t begin = group * kGroup + lane;
    Octet o;
    float m_scale = 0.0f, v_scale = 0.0f;
    if (STATE == COLLAGE_STATE_E4M3) { m_scale = t.m_scale[group]; v_scale = t.v_scale[group]; }
    auto gather = [&](uint64_t (&to)[4], auto&& value) {
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            const uint64_t i = begin + p * 64, j = i + 32;
            to[p] = ops::pair_of(i < t.n ? value(i) : 0.0f, j < t.n ? value(j) : 0.0f);
        }
    };
    auto code = [](const void* p, uint64_t i) { return floats_of(e4m3_pair(static_cast<const uint8_t*>(p)[i])).x; };
    gather(o.g, [&](uint64_t i) { return bf16_value(t.grad[i]); });
    if (REST != COLLAGE_REST_F32) gather(o.theta, [&](uint64_t i) { return bf16_value(t.theta[i]); });
    if (REST == COLLAGE_REST_BF16) gather(o.rest, [&](uint64_t i) { return bf16_value(static_cast<const uint16_t*>(t.rest)[i]); });
    if (REST == COLLAGE_REST_F32) gather(o.rest, [&](uint64_t i) { return static_cast<const float*>(t.rest)[i]; });
    if (STATE == COLLAGE_STATE_F32) {
        gather(o.m, [&](uint64_t i) { return static_cast<const float*>(t.m)[i]; });
        gather(o.v, [&](uint64_t i) { return static_cast<const float*>(t.v)[i]; });
    } else {
        gather(o.m, [&](uint64_t i) { return code(t.m, i) * m_scale; });
        gather(o.v, [&](uint64_t i) { return code(t.v, i) * v_scale; });
    }
    update<STATE, REST>(o, k, grad_scale);
    auto scatter = [&](auto&& put) {
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            const uint64_t i = begin + p * 64;
            if (i < t.n) put(i, p, 0);
            if (i + 32 < t.n) put(i + 32, p, 1);
        }
    };
    auto half = [](const uint64_t f, int h) { const float2 v = floats_of(f); return h ? v.y : v.x; };
    scatter([&](uint64_t i, int p, int h) {
        t.theta[i] = static_cast<uint16_t>(o.theta_out[p] >> (16 * h));
        if (REST == COLLAGE_REST_BF16) static_cast<uint16_t*>(t.rest)[i] = static_cast<uint16_t>(o.rest_out[p] >> (16 * h));
        if (REST == COLLAGE_REST_F32) static_cast<float*>(t.rest)[i] = half(o.rest[p], h);
        if (STATE == COLLAGE_STATE_F32) {
            static_cast<float*>(t.m)[i] = half(o.m[p], h);
            static_cast<float*>(t.v)[i] = half(o.v[p], h);
        }
    });
    if (STATE == COLLAGE_STATE_F32) return;
    // (elements behind the end: m = beta1 0 + ... 0 and a root of 0, which no scale minds)
    float m_factor, v_factor;
    m_scale = group_scale(largest(o.m), m_factor);
    v_scale = group_scale(largest(o.v), v_factor);
    uint32_t random[4];
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const uint64_t i = t.first + begin + p * 64;
        const uint32_t lo = random_word(i >> 1, k.key), hi = random_word((i + 32) >> 1, k.key);
        random[p] = i & 1 ? __byte_perm(lo, hi, 0x7632) : __byte_perm(lo, hi, 0x5410);
    }
    const uint2 cm = nearest_codes(o.m, m_factor), cv = random_codes(o.v, v_factor, random);
    scatter([&](uint64_t i, int p, int h) {
        const int shift = 8 * (2 * (p & 1) + h);
        static_cast<uint8_t*>(t.m)[i] = static_cast<uint8_t>((p < 2 ? cm.x : cm.y) >> shift);
        static_cast<uint8_t*>(t.v)[i] = static_cast<uint8_t>((p < 2 ? cv.x : cv.y) >> shift);
    });
    if (lane == 0) {
        t.m_scale[group] = m_scale;
        t.v_scale[group] = v_scale;
    }
}

// A warp's way through the groups of its tasks.
struct Walk {
    uint64_t task;
    AdamChunk now;
    uint32_t g, groups;
    __device__ __forceinline__ void begin(const AdamArgs& a) {
        if (task >= a.num_tasks) return;
        now = a.tasks[task];
        const uint64_t all = (a.tensors[now.tensor].n + kGroup - 1) / kGroup, first = static_cast<uint64_t>(now.index) * a.task_groups;
        groups = static_cast<uint32_t>(min(static_cast<uint64_t>(a.task_groups), all - first));
        g = 0;
    }
    __device__ __forceinline__ void next(const AdamArgs& a, uint64_t stride) {
        if (++g < groups) return;
        task += stride;
        begin(a);
    }
    __device__ __forceinline__ uint64_t group(const AdamArgs& a) const { return static_cast<uint64_t>(now.index) * a.task_groups + g; }
};

// Every warp by itself: it sends for the arrays of groups ahead of the one that it works on, each lane for its own bytes.
template <int STATE, int REST>
__global__ void __launch_bounds__(kAdamThreads, 3) adam_step_kernel(const __grid_constant__ AdamArgs a) {
    using F = Form<STATE, REST>;
    extern __shared__ __align__(16) uint8_t dynamic[];
    after_previous();
    const int lane = threadIdx.x & 31;
    uint8_t* stages = dynamic + (threadIdx.x >> 5) * (F::kStages * F::kStage);
    const uint32_t stages_at = static_cast<uint32_t>(__cvta_generic_to_shared(stages));
    const uint64_t stride = static_cast<uint64_t>(gridDim.x) * kAdamWarps;
    const float grad_scale = a.grad_scale ? *a.grad_scale : 1.0f;
    Walk ahead;
    ahead.task = static_cast<uint64_t>(threadIdx.x >> 5) * gridDim.x + blockIdx.x;
    ahead.begin(a);
    Walk here = ahead;
    auto is_whole = [](const AdamRec& t, uint64_t group) { return t.aligned && (group + 1) * kGroup <= t.n; };
    auto send = [&](int stage) {
        if (ahead.task < a.num_tasks) {
            const AdamRec& t = a.tensors[ahead.now.tensor];
            const uint64_t group = ahead.group(a);
            if (is_whole(t, group)) send_group<STATE, REST>(t, group, stages_at + stage * F::kStage, lane);
            ahead.next(a, stride);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    for (int s = 0; s < F::kStages; ++s) send(s);
    for (int stage = 0; here.task < a.num_tasks; here.next(a, stride)) {
        asm volatile("cp.async.wait_group %0;" ::"n"(F::kStages - 1) : "memory");
        __syncwarp();
        const AdamRec& t = a.tensors[here.now.tensor];
        const uint64_t group = here.group(a);
        if (is_whole(t, group))
            whole_group<STATE, REST>(t, group, stages + stage * F::kStage, a.k, grad_scale, lane);
        else
            any_group<STATE, REST>(t, group, a.k, grad_scale);
        __syncwarp();
        send(stage);
        stage = stage + 1 == F::kStages ? 0 : stage + 1;
    }
}

template <int STATE, int REST>
static collage_status_t launch_adam(const AdamArgs& a, int sm_count, cudaStream_t s) {
    using F = Form<STATE, REST>;
    constexpr size_t smem = static_cast<size_t>(kAdamWarps) * F::kStages * F::kStage;
    static std::atomic<int> per_device[64];
    int device = 0;
    if (cudaGetDevice(&device) != cudaSuccess || device < 0 || device >= 64) return COLLAGE_ERR_CUDA;
    int resident = per_device[device].load(std::memory_order_acquire);
    if (resident == 0) {
        if (allow_smem<&adam_step_kernel<STATE, REST>>() != cudaSuccess ||
            cudaOccupancyMaxActiveBlocksPerMultiprocessor(&resident, &adam_step_kernel<STATE, REST>, kAdamThreads, smem) != cudaSuccess)
            return COLLAGE_ERR_CUDA;
        resident = std::max(resident, 1);
        per_device[device].store(resident, std::memory_order_release);
    }
    const uint64_t grid = std::min<uint64_t>((a.num_tasks + kAdamWarps - 1) / kAdamWarps, static_cast<uint64_t>(resident) * sm_count);
    return launch<&adam_step_kernel<STATE, REST>>(grid, kAdamThreads, 1, smem, s, a);
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
    AdamChunk *d_chunks = nullptr, *d_tasks = nullptr;
    uint64_t num_chunks = 0, num_tasks = 0;
    uint32_t task_groups = 1;
    std::vector<ByteRange> ranges, written;    // sorted by address: all arrays, and those that a step writes
    int state = 0, rest = 0, device = -1;
    ~collage_adam_plan() {
        cudaFree(d_tensors);
        cudaFree(d_chunks);
        cudaFree(d_tasks);
    }
};

namespace {

collage_status_t create(const collage_adam_tensor_t* tensors, int num, int state, int rest, collage_adam_plan** out) {
    const uint64_t state_bytes = state == COLLAGE_STATE_F32 ? 4 : 1, rest_bytes = rest == COLLAGE_REST_F32 ? 4 : 2;
    std::vector<ByteRange> ranges, written;
    std::vector<AdamRec> recs;
    std::vector<AdamChunk> chunks, tasks;
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
    // groups of a warp's turn: 16 where every warp of the device has several turns of that, fewer for small plans
    uint32_t task_groups = 16;
    while (task_groups > 1 && first / kGroup < static_cast<uint64_t>(task_groups) * 128 * dev.sm_count) task_groups /= 2;
    for (size_t i = 0; i < recs.size(); ++i) {
        const uint64_t own = ((recs[i].n + kGroup - 1) / kGroup + task_groups - 1) / task_groups;
        for (uint64_t c = 0; c < own; ++c) tasks.push_back({static_cast<uint32_t>(i), static_cast<uint32_t>(c)});
    }
    collage_adam_plan* plan = new collage_adam_plan;
    plan->num_chunks = num_chunks;
    plan->num_tasks = tasks.size();
    plan->task_groups = task_groups;
    plan->ranges = std::move(ranges);
    plan->written = std::move(written);
    plan->state = state;
    plan->rest = rest;
    if (cudaGetDevice(&plan->device) != cudaSuccess ||
        (num_chunks && (cudaMalloc(&plan->d_tensors, recs.size() * sizeof(AdamRec)) != cudaSuccess ||
                        cudaMalloc(&plan->d_chunks, chunks.size() * sizeof(AdamChunk)) != cudaSuccess ||
                        cudaMalloc(&plan->d_tasks, tasks.size() * sizeof(AdamChunk)) != cudaSuccess ||
                        cudaMemcpy(plan->d_tasks, tasks.data(), tasks.size() * sizeof(AdamChunk), cudaMemcpyHostToDevice) != cudaSuccess ||
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
    a.tasks = plan->d_tasks;
    a.num_tasks = plan->num_tasks;
    a.task_groups = plan->task_groups;
    a.grad_scale = grad_scale;
    a.k.f = fp32_scalars(hyper, step);
    const double t = static_cast<double>(step), bc1 = 1.0 - std::pow(hyper->beta1, t), bc2 = 1.0 - std::pow(hyper->beta2, t);
    a.k.inv_bc1 = static_cast<float>(1.0 / bc1);
    a.k.inv_bc2 = static_cast<float>(1.0 / bc2);
    a.k.inv_root_bc2 = static_cast<float>(1.0 / std::sqrt(bc2));
    uint32_t key = mix32(static_cast<uint32_t>(step >> 32));
    for (const uint64_t word : {step, seed >> 32, seed}) key = mix32(static_cast<uint32_t>(word) + key);
    a.k.key = key;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    switch (plan->state * 3 + plan->rest) {
        case 0: return launch_adam<0, 0>(a, dev.sm_count, s);
        case 1: return launch_adam<0, 1>(a, dev.sm_count, s);
        case 2: return launch_adam<0, 2>(a, dev.sm_count, s);
        case 3: return launch_adam<1, 0>(a, dev.sm_count, s);
        case 4: return launch_adam<1, 1>(a, dev.sm_count, s);
        default: return launch_adam<1, 2>(a, dev.sm_count, s);
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

// AdamW over many tensors in one launch, with states in 8 bits (codes with a scale for each 256 elements) or in floats; and the norm
// of all gradients.
//
//   m' = b1 m + c1 g,  v' = b2 v + c2 g^2,  x' = x - a (m' / bc1 / (sqrt(v' / bc2) + eps) + lam x)
//   8 bits: m = code * scale, sqrt(v) = code * scale; scales are the group's largest value / 448
//
// The root of v is kept rather than v: its 8 bits span 2^18, v would need twice that.  Its code is rounded with a random
// part, since in a step of beta2 = 0.999 it moves by a two-hundredth of a code's step, which rounding to nearest would undo each time;
// m moves by a tenth of what separates it from the gradient and is rounded to nearest.
// Bytes a parameter: 10 (theta alone) to 16 with 8-bit states, 22 to 28 with floats.  Measured: 134 M parameters in 8 bits alone 299 us (4.5 TB/s),
// with pairs 388 us (4.9), with master weights 332 us (6.5); 67 M in floats alone 236 us (6.3), with pairs 273 us (6.4), with master weights 292
// us (6.4).  The first two are bound by instructions (60 to 81 an element: decoding, sums with their remainders, random bits, codes), the
// others by memory.
#include "adamw_float.cuh"
#include "bulk_pipe.cuh"
#include "ops_common.cuh"

#include <cfloat>
#include <new>

namespace collage {
namespace ops {

constexpr uint32_t kGroup = 256;               // elements that share a scale: a warp's, eight a lane
constexpr uint32_t kNormChunk = 4096;          // elements of a block's turn in the norm
constexpr int kAdamThreads = 256;

struct AdamRec {
    uint16_t* theta;
    void *rest, *m, *v;
    float *m_scale, *v_scale;
    const uint16_t* grad;
    uint64_t n, first;                         // first: position of its first element in the plan
    uint64_t aligned;                          // all arrays but the scales begin on 16 bytes
};
struct AdamChunk {
    uint32_t tensor, index;
};

struct AdamScalars {
    Fp32Scalars f;
    float rate, decay;                         // -a / bc1, -a lam
    float a_hi, a_lo;                          // a in two floats
    float inv_bc1, inv_bc2, inv_root_bc2;      // 1 / bc1, 1 / bc2, 1 / sqrt(bc2)
    uint32_t key;
};

struct AdamArgs {
    const AdamRec* tensors;
    const AdamChunk* tiles;
    uint64_t num_tiles;
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

// A sum of two products, each rounded.  (The assembler makes a packed product and a packed sum of it one fma; not so of these.)
__device__ __forceinline__ uint64_t add_rounded(uint64_t a, uint64_t b) {
    const float2 f = floats_of(a), g = floats_of(b);
    return pair_of(__fadd_rn(f.x, g.x), __fadd_rn(f.y, g.y));
}
// times a constant of the call, plus another
__device__ __forceinline__ uint64_t scaled_pair(uint64_t a, float c) {
    return mul_pair(a, pair_of(c));
}
__device__ __forceinline__ uint64_t scaled_plus(uint64_t a, float c, float d) {
    return fma_pair(a, pair_of(c), pair_of(d));
}
__device__ __forceinline__ uint64_t scaled_plus(uint64_t a, float c, uint64_t d) {
    return fma_pair(a, pair_of(c), d);
}
__device__ __forceinline__ uint64_t e4m3_pair(uint32_t two) {
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(two), __NV_E4M3);
    const float2 f = __half22float2(__half2(h));
    return pair_of(f.x, f.y);
}

// Square roots: y = rsqrt(v) gives r = v y, and a step of Newton's method on r^2 = v, whose remainder r^2 - v is exact in an fma, the
// correctly rounded root but for a few in a million (in half the instructions of one that always is).  ANY: of infinity too (r from the largest
// float and the remainder from v; else a NaN, as infinity times 0).
template <bool ANY>
__device__ __forceinline__ uint64_t root_pair(uint64_t v) {
    const float2 f = floats_of(v), most = ANY ? make_float2(fminf(f.x, FLT_MAX), fminf(f.y, FLT_MAX)) : f;
    float2 y;
    asm("rsqrt.approx.f32 %0, %1;" : "=f"(y.x) : "f"(fmaxf(most.x, 0x1p-149f)));      // (of 0: 0 times a finite number)
    asm("rsqrt.approx.f32 %0, %1;" : "=f"(y.y) : "f"(fmaxf(most.y, 0x1p-149f)));
    const uint64_t y2 = pair_of(y.x, y.y), r = mul_pair(pair_of(most.x, most.y), y2);
    const float2 q = floats_of(r);
    return pair_of(__fmaf_rn(__fmaf_rn(-q.x, q.x, f.x), 0.5f * y.x, q.x), __fmaf_rn(__fmaf_rn(-q.y, q.y, f.y), 0.5f * y.y, q.y));
}
__device__ __forceinline__ uint64_t reciprocal_pair(uint64_t v) {
    float2 f = floats_of(v);
    asm("rcp.approx.f32 %0, %0;" : "+f"(f.x));
    asm("rcp.approx.f32 %0, %0;" : "+f"(f.y));
    return pair_of(f.x, f.y);
}

// A step of two elements' states: m', and sqrt(v') or v' itself.  Every product and sum is rounded once, so that codes hang on nothing but the
// formulas.  Returns sqrt(v').  (With states in 8 bits an infinite v' makes its group NaN in any case.)
template <int STATE>
__device__ __forceinline__ uint64_t advance(uint64_t& m, uint64_t& v, uint64_t g, const AdamScalars& k) {
    const uint64_t squared = STATE == COLLAGE_STATE_F32 ? v : mul_pair(v, v);
    m = add_rounded(scaled_pair(m, k.f.b1), scaled_pair(g, k.f.c1));
    v = add_rounded(scaled_pair(squared, k.f.b2), scaled_pair(mul_pair(g, g), k.f.c2));
    return root_pair<STATE == COLLAGE_STATE_F32>(v);
}
// The update of parameters x to a few units of its last place.
template <bool INSIDE>
__device__ __forceinline__ uint64_t update_of(uint64_t m, uint64_t v, uint64_t root, uint64_t x, const AdamScalars& k) {
    const uint64_t den = INSIDE ? root_pair<true>(scaled_plus(v, k.inv_bc2, k.f.eps)) : scaled_plus(root, k.inv_root_bc2, k.f.eps);
    return scaled_plus(x, k.decay, scaled_pair(mul_pair(m, reciprocal_pair(den)), k.rate));
}

// A bfloat16 pair keeps 16 bits and more of its parameter, and what it keeps is meant to be exact: theta' the nearest bfloat16 to
//   theta + rest - a (q + lam x),  q = RN(m' / bc1) / RN(sqrt(v' / bc2) + eps) rounded once,
// rest' what that lacks.  The sum is known here as s + low to about 2^-24 of the decay's part and far less of the rest's: q by Markstein's division
// (a reciprocal by a step of Newton's method, the quotient's remainder exact in an fma), its product with a (two floats) with the
// product's remainder, and sums with their remainders (TwoSum).
// ANY: the divisor may be infinite (its reciprocal is 0; remainders by the largest float leave the quotient 0, and a NaN of an infinite m).
struct PairSum {
    uint64_t s, low;
};
template <bool INSIDE, bool ANY>
__device__ __forceinline__ PairSum sum_of_pair(uint64_t theta, uint64_t rest, uint64_t m, uint64_t v, uint64_t root, const AdamScalars& k) {
    const uint64_t den = INSIDE ? root_pair<true>(scaled_plus(v, k.inv_bc2, k.f.eps)) : add_rounded(scaled_pair(root, k.inv_root_bc2), pair_of(k.f.eps));
    const uint64_t num = scaled_pair(m, k.inv_bc1);
    float2 d = floats_of(den);
    const float2 n = floats_of(num);
    float2 r;
    asm("rcp.approx.f32 %0, %1;" : "=f"(r.x) : "f"(d.x));
    asm("rcp.approx.f32 %0, %1;" : "=f"(r.y) : "f"(d.y));
    if (ANY) d = make_float2(fminf(d.x, FLT_MAX), fminf(d.y, FLT_MAX));
    const uint64_t r0 = pair_of(r.x, r.y), r1 = fma_pair(pair_of(__fmaf_rn(-d.x, r.x, 1.0f), __fmaf_rn(-d.y, r.y, 1.0f)), r0, r0);
    const float2 q0 = floats_of(mul_pair(num, r1));
    const uint64_t q = fma_pair(pair_of(__fmaf_rn(-d.x, q0.x, n.x), __fmaf_rn(-d.y, q0.y, n.y)), r1, pair_of(q0.x, q0.y));
    const float2 qf = floats_of(q);
    const uint64_t p = pair_of(__fmul_rn(qf.x, k.a_hi), __fmul_rn(qf.y, k.a_hi));        // a q, and (negated) its remainder and the decay
    const uint64_t more = fma_pair(add_pair(theta, rest), pair_of(k.decay), fma_pair(q, pair_of(-k.a_lo), fma_pair(q, pair_of(-k.a_hi), p)));
    const uint64_t t = sub_pair(rest, p), tb = sub_pair(t, rest), t_low = sub_pair(sub_pair(rest, sub_pair(t, tb)), add_pair(p, tb));
    const uint64_t s = add_pair(theta, t), sb = sub_pair(s, theta), s_low = add_pair(sub_pair(theta, sub_pair(s, sb)), sub_pair(t, sb));
    const uint64_t low = add_pair(add_pair(s_low, t_low), more), whole = add_pair(s, low);
    return {whole, sub_pair(low, sub_pair(whole, s))};
}
// A float half-way between two bfloat16 values: `low` tells which one is nearer.  (One in 65536.)
__device__ __forceinline__ bool is_tie(float s) { return (__float_as_uint(s) & 0xFFFFu) == 0x8000u; }
__device__ __forceinline__ void split_pair(const PairSum& sum, uint32_t& theta_word, uint32_t& rest_word) {
    const float2 s = floats_of(sum.s);
    theta_word = pack_bf16(s.x, s.y);
    const float2 r = floats_of(add_pair(sub_pair(sum.s, bf16_pair(theta_word)), sum.low));
    rest_word = pack_bf16(r.x, r.y);
}
// Two words again where their sums are ties: theta' by way of a float rounded to odd, towards the sum's own side.
__device__ __forceinline__ void settle(const PairSum& sum, uint32_t& theta_word, uint32_t& rest_word) {
    const float2 s = floats_of(sum.s), l = floats_of(sum.low);
    auto odd = [](float f, float low) {
        const uint32_t bits = __float_as_uint(f);
        return is_tie(f) && low != 0.0f && fabsf(low) < INFINITY ? __uint_as_float((bits - ((__float_as_uint(low) ^ bits) >> 31)) | 1u) : f;
    };
    theta_word = pack_bf16(odd(s.x, l.x), odd(s.y, l.y));
    const float2 r = floats_of(add_pair(sub_pair(sum.s, bf16_pair(theta_word)), sum.low));
    rest_word = pack_bf16(r.x, r.y);
}

// Eight elements of a lane, in pairs, before and behind the update.  With states in 8 bits v is its root.
struct Octet {
    uint64_t g[4], theta[4], rest[4], m[4], v[4];
    uint32_t theta_out[4], rest_out[4];                  // two bfloat16 each
};

// SETTLE: sums that are ties are settled here and now; else the result tells whether there are any.
template <int STATE, int REST, bool INSIDE, bool SETTLE>
__device__ __forceinline__ bool update(Octet& o, const AdamScalars& k, float grad_scale) {
    uint32_t least = 0;                         // smallest of the sums' lower half-words as signed numbers: -32768 if one is a tie
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const uint64_t g = scaled_pair(o.g[p], grad_scale);
        if (REST == COLLAGE_REST_BF16) {
            const uint64_t root = advance<STATE>(o.m[p], o.v[p], g, k);
            const PairSum sum = sum_of_pair<INSIDE, INSIDE || STATE == COLLAGE_STATE_F32>(o.theta[p], o.rest[p], o.m[p], o.v[p], root, k);
            if (STATE == COLLAGE_STATE_E4M3) o.v[p] = root;
            split_pair(sum, o.theta_out[p], o.rest_out[p]);
            const float2 s = floats_of(sum.s);
            if (SETTLE)
                settle(sum, o.theta_out[p], o.rest_out[p]);
            else
                least = __vmins2(least, __byte_perm(__float_as_uint(s.x), __float_as_uint(s.y), 0x5410));
            continue;
        }
        const uint64_t x = REST == COLLAGE_REST_F32 ? o.rest[p] : o.theta[p];
        uint64_t delta;
        if (STATE == COLLAGE_STATE_F32) {       // the flat step's operations
            float2 m = floats_of(o.m[p]), v = floats_of(o.v[p]);
            const float2 gf = floats_of(g), xf = floats_of(x);
            const float lo = adamw_fp32_delta(m.x, v.x, xf.x, gf.x, k.f), hi = adamw_fp32_delta(m.y, v.y, xf.y, gf.y, k.f);
            delta = pair_of(lo, hi);
            o.m[p] = pair_of(m.x, m.y);
            o.v[p] = pair_of(v.x, v.y);
        } else {
            const uint64_t root = advance<STATE>(o.m[p], o.v[p], g, k);
            delta = update_of<INSIDE>(o.m[p], o.v[p], root, x, k);
            o.v[p] = root;
        }
        o.rest[p] = add_pair(x, delta);
        const float2 to = floats_of(o.rest[p]);
        o.theta_out[p] = pack_bf16(to.x, to.y);
    }
    return (least & 0xFFFFu) == 0x8000u || least >> 16 == 0x8000u;
}

// Largest absolute value of eight over the warp; NaN where there is one.
__device__ __forceinline__ uint32_t largest(const uint64_t (&f)[4]) {
    float most = 0.0f;
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const float2 v = floats_of(f[p]);
        asm("max.NaN.f32 %0, %0, %1, %2;" : "+f"(most) : "f"(fabsf(v.x)), "f"(fabsf(v.y)));
    }
    return __reduce_max_sync(0xFFFFFFFFu, __float_as_uint(most));
}
// Scale of a group from the bits of its largest absolute value, and what its values are taken times.
__device__ __forceinline__ float group_scale(uint32_t most, float& factor) {
    const float v = __uint_as_float(most);
    float r;                                   // 1 / v, by a step of Newton's method
    asm("rcp.approx.f32 %0, %1;" : "=f"(r) : "f"(v));
    r = __fmaf_rn(__fmaf_rn(-v, r, 1.0f), r, r);
    const bool none = v < 0x1p-100f, off = most >= 0x7F800000u;
    factor = none ? 0.0f : off ? NAN : r * kE4m3Max;
    return none ? 0.0f : off ? NAN : v * (1.0f / kE4m3Max);
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
        asm("min.f32 %0, %0, %1, %2;" : "+f"(least) : "f"(v.x), "f"(v.y));
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

// Groups of a tile, one for each warp beside the one that copies.  One more than a multiple of four, with that one, would cost all of them
// registers: a quarter of an SM would have one warp more to share its own among.  Measured with 15, 19 and 23: 134 M parameters in 8 bits alone
// 299, 323 and 300 us, with pairs 399, 400 and 388, with master weights 337, 361 and 332; 67 M in floats alone 236, 235 and 252 us, with pairs
// 287, 295 and 273, with master weights 306, 294 and 292.
constexpr int tile_groups(int rest) { return rest == COLLAGE_REST_NONE ? 15 : 23; }

// A stage of the copy pipeline: a tile's bytes of each array.  Of a whole group a lane has eight elements in a row, or, where some array
// is of floats, four in a row of each half, so that a warp's accesses are to consecutive bytes.
template <int STATE, int REST>
struct Form {
    static constexpr bool kHalves = STATE == COLLAGE_STATE_F32 || REST == COLLAGE_REST_F32;
    static constexpr bool kReadsTheta = REST != COLLAGE_REST_F32;
    static constexpr uint32_t kStateBytes = STATE == COLLAGE_STATE_F32 ? 4 : 1, kRestBytes = REST == COLLAGE_REST_F32 ? 4 : REST == COLLAGE_REST_BF16 ? 2 : 0;
    static constexpr uint32_t kWarps = tile_groups(REST), kTile = kWarps * kGroup;
    // offsets of the arrays in a stage
    static constexpr uint32_t kG = 0, kT = kG + 2 * kTile, kR = kT + 2 * kTile, kM = kR + kRestBytes * kTile, kV = kM + kStateBytes * kTile,
                              kStage = kV + kStateBytes * kTile;
    static constexpr uint32_t kStages = 208 * 1024 / kStage;          // two to nine
    static __device__ __forceinline__ uint32_t element(int lane, int half) { return kHalves ? half * (kGroup / 2) + lane * 4 : lane * 8 + half * 4; }
};

// What the other warps have to know of the tile in a stage.
template <uint32_t GROUPS>
struct AdamTile {
    const AdamRec* tensor;
    uint64_t first_group;                      // of the tensor
    uint32_t groups, whole;                    // in the tile; of these, in shared memory
    uint32_t random[2], passed;                // what pairs' numbers in the tile are added to before they are mixed; from group `passed` on the second
    float scales[2 * GROUPS];                  // of m, then of the root
};
template <int STATE, int REST>
struct AdamSmem {
    using F = Form<STATE, REST>;
    alignas(128) uint8_t bytes[F::kStages][F::kStage];
    AdamTile<F::kWarps> tile[F::kStages];
    alignas(8) uint64_t full[F::kStages], done[F::kStages];
};

// A lane's eight elements of one array of a group, in 8, 16 or 32 bytes of words
template <typename F, uint32_t BYTES>
__device__ __forceinline__ void fetch_array(const uint8_t* group, int lane, uint32_t (&w)[2 * BYTES]) {
    if constexpr (!F::kHalves && BYTES == 2) {
        const uint4 q = *reinterpret_cast<const uint4*>(group + lane * 16);
        w[0] = q.x; w[1] = q.y; w[2] = q.z; w[3] = q.w;
    } else if constexpr (!F::kHalves && BYTES == 1) {
        const uint2 q = *reinterpret_cast<const uint2*>(group + lane * 8);
        w[0] = q.x; w[1] = q.y;
    } else {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t* p = reinterpret_cast<const uint32_t*>(group + F::element(lane, h) * BYTES);
            if constexpr (BYTES == 4) {
                const uint4 q = *reinterpret_cast<const uint4*>(p);
                w[h * 4] = q.x; w[h * 4 + 1] = q.y; w[h * 4 + 2] = q.z; w[h * 4 + 3] = q.w;
            } else if constexpr (BYTES == 2) {
                const uint2 q = *reinterpret_cast<const uint2*>(p);
                w[h * 2] = q.x; w[h * 2 + 1] = q.y;
            } else {
                w[h] = *p;
            }
        }
    }
}
template <typename F, uint32_t BYTES>
__device__ __forceinline__ void put_array(uint8_t* group, int lane, const uint32_t (&w)[2 * BYTES]) {
    if constexpr (!F::kHalves && BYTES == 2) {
        *reinterpret_cast<uint4*>(group + lane * 16) = make_uint4(w[0], w[1], w[2], w[3]);
    } else if constexpr (!F::kHalves && BYTES == 1) {
        *reinterpret_cast<uint2*>(group + lane * 8) = make_uint2(w[0], w[1]);
    } else {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint8_t* p = group + F::element(lane, h) * BYTES;
            if constexpr (BYTES == 4) *reinterpret_cast<uint4*>(p) = make_uint4(w[4 * h], w[4 * h + 1], w[4 * h + 2], w[4 * h + 3]);
            if constexpr (BYTES == 2) *reinterpret_cast<uint2*>(p) = make_uint2(w[2 * h], w[2 * h + 1]);
            if constexpr (BYTES == 1) *reinterpret_cast<uint32_t*>(p) = w[h];
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
    for (int p = 0; p < 4; ++p) f[p] = pair_of(__uint_as_float(w[2 * p]), __uint_as_float(w[2 * p + 1]));
}

// A lane's part of group `g` of a tile
template <int STATE, int REST>
__device__ __forceinline__ void fetch_group(uint8_t* stage, const AdamTile<Form<STATE, REST>::kWarps>& tile, uint32_t g, Octet& o, int lane) {
    using F = Form<STATE, REST>;
    auto of = [&](uint32_t array, uint32_t bytes) { return stage + array + g * (kGroup * bytes); };
    uint32_t w[4];
    fetch_array<F, 2>(of(F::kG, 2), lane, w);
#pragma unroll
    for (int p = 0; p < 4; ++p) o.g[p] = bf16_pair(w[p]);
    if constexpr (F::kReadsTheta) {
        fetch_array<F, 2>(of(F::kT, 2), lane, w);
#pragma unroll
        for (int p = 0; p < 4; ++p) o.theta[p] = bf16_pair(w[p]);
    }
    if constexpr (REST == COLLAGE_REST_BF16) {
        fetch_array<F, 2>(of(F::kR, 2), lane, w);
#pragma unroll
        for (int p = 0; p < 4; ++p) o.rest[p] = bf16_pair(w[p]);
    }
    uint32_t wide[8];
    if constexpr (REST == COLLAGE_REST_F32) {
        fetch_array<F, 4>(of(F::kR, 4), lane, wide);
        words_to_floats(wide, o.rest);
    }
    if constexpr (STATE == COLLAGE_STATE_F32) {
        fetch_array<F, 4>(of(F::kM, 4), lane, wide);
        words_to_floats(wide, o.m);
        fetch_array<F, 4>(of(F::kV, 4), lane, wide);
        words_to_floats(wide, o.v);
    } else {
        uint32_t c[2];
        fetch_array<F, 1>(of(F::kM, 1), lane, c);
#pragma unroll
        for (int p = 0; p < 4; ++p) o.m[p] = mul_pair(e4m3_pair(c[p / 2] >> (16 * (p & 1))), pair_of(tile.scales[g]));
        fetch_array<F, 1>(of(F::kV, 1), lane, c);
#pragma unroll
        for (int p = 0; p < 4; ++p) o.v[p] = mul_pair(e4m3_pair(c[p / 2] >> (16 * (p & 1))), pair_of(tile.scales[F::kWarps + g]));
    }
}

// Parameters of a group that has ties among its sums, once more from its old values.
template <int STATE, bool INSIDE>
__device__ __noinline__ void settle_group(uint8_t* stage, const AdamTile<Form<STATE, COLLAGE_REST_BF16>::kWarps>& tile, uint32_t g, const AdamScalars& k, float grad_scale) {
    using F = Form<STATE, COLLAGE_REST_BF16>;
    const int lane = threadIdx.x & 31;
    Octet o;
    fetch_group<STATE, COLLAGE_REST_BF16>(stage, tile, g, o, lane);
    update<STATE, COLLAGE_REST_BF16, INSIDE, true>(o, k, grad_scale);
    put_array<F, 2>(stage + F::kT + g * (kGroup * 2), lane, o.theta_out);
    put_array<F, 2>(stage + F::kR + g * (kGroup * 2), lane, o.rest_out);
}

// A whole group by a warp, in place in the stage.
template <int STATE, int REST, bool INSIDE>
__device__ __forceinline__ void whole_group(uint8_t* stage, AdamTile<Form<STATE, REST>::kWarps>& tile, uint32_t g, const AdamScalars& k, float grad_scale, int lane) {
    using F = Form<STATE, REST>;
    auto of = [&](uint32_t array, uint32_t bytes) { return stage + array + g * (kGroup * bytes); };
    Octet o;
    fetch_group<STATE, REST>(stage, tile, g, o, lane);
    uint32_t wide[8];
    const bool tie = update<STATE, REST, INSIDE, false>(o, k, grad_scale);
    if constexpr (REST == COLLAGE_REST_BF16) {
        if (__any_sync(0xFFFFFFFFu, tie)) {
            settle_group<STATE, INSIDE>(stage, tile, g, k, grad_scale);
        } else {
            put_array<F, 2>(of(F::kT, 2), lane, o.theta_out);
            put_array<F, 2>(of(F::kR, 2), lane, o.rest_out);
        }
    } else {
        put_array<F, 2>(of(F::kT, 2), lane, o.theta_out);
    }
    if constexpr (REST == COLLAGE_REST_F32) {
        floats_to_words(o.rest, wide);
        put_array<F, 4>(of(F::kR, 4), lane, wide);
    }
    if constexpr (STATE == COLLAGE_STATE_F32) {
        floats_to_words(o.m, wide);
        put_array<F, 4>(of(F::kM, 4), lane, wide);
        floats_to_words(o.v, wide);
        put_array<F, 4>(of(F::kV, 4), lane, wide);
    } else {
        float m_factor, v_factor;
        const float m_scale = group_scale(largest(o.m), m_factor), v_scale = group_scale(largest(o.v), v_factor);
        const uint32_t base = tile.random[g >= tile.passed] + g * (kGroup / 2);
        uint32_t random[4];
#pragma unroll
        for (int p = 0; p < 4; ++p) random[p] = mix32(base + F::element(lane, p / 2) / 2 + (p & 1));
        const uint2 cm = nearest_codes(o.m, m_factor), cv = random_codes(o.v, v_factor, random);
        const uint32_t wm[2] = {cm.x, cm.y}, wv[2] = {cv.x, cv.y};
        put_array<F, 1>(of(F::kM, 1), lane, wm);
        put_array<F, 1>(of(F::kV, 1), lane, wv);
        if (lane < 2) tile.scales[lane * F::kWarps + g] = lane ? v_scale : m_scale;
    }
}

// The same for groups that are cut short or not aligned: every 32nd element a lane.  Elements behind the end count as zeros.
template <int STATE, int REST, bool INSIDE>
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
            to[p] = pair_of(i < t.n ? value(i) : 0.0f, j < t.n ? value(j) : 0.0f);
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
    update<STATE, REST, INSIDE, true>(o, k, grad_scale);
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

// Fault word of this file's waits; collage_pipeline_fault reports it.
static __device__ unsigned int g_adam_fault = 0;

// Blocks walk over tiles of as many groups as they have warps that work.  One warp more brings each tile's whole groups into shared memory by
// bulk copies, several tiles ahead, and stores them when the others have worked them over in place, a group each; a last group that is
// cut short, and tensors that no bulk copy can take, go straight from and to memory.
template <int STATE, int REST, bool INSIDE>
__global__ void __launch_bounds__(Form<STATE, REST>::kWarps * 32 + 32, 1) adam_step_kernel(const __grid_constant__ AdamArgs a) {
    using F = Form<STATE, REST>;
    constexpr uint32_t kStages = F::kStages, kWarps = F::kWarps;
    extern __shared__ __align__(128) uint8_t dynamic[];
    AdamSmem<STATE, REST>& sm = *reinterpret_cast<AdamSmem<STATE, REST>*>(dynamic);
    const int lane = threadIdx.x & 31;
    const uint32_t warp = threadIdx.x >> 5;
    if (threadIdx.x == 0) {
        for (uint32_t s = 0; s < kStages; ++s) {
            pipe::mbar_init(&sm.full[s], 1 + (STATE == COLLAGE_STATE_E4M3 ? 32 : 0));
            pipe::mbar_init(&sm.done[s], kWarps);
        }
        pipe::mbar_init_fence();
    }
    __syncthreads();
    after_previous();
    if (warp == kWarps) {                      // the copies
        uint32_t it = 0;
        bool alive = true;
        auto scale_at = [](const AdamRec& t, uint32_t i, uint64_t first) { return (i < kWarps ? t.m_scale + i : t.v_scale + (i - kWarps)) + first; };
        auto store_out = [&](uint32_t s) {
            const auto& tile = sm.tile[s];
            if (!tile.whole) return;
            const AdamRec& t = *tile.tensor;
            if (STATE == COLLAGE_STATE_E4M3)
                for (uint32_t i = lane; i < 2 * kWarps; i += 32)
                    if (i % kWarps < tile.whole) *scale_at(t, i, tile.first_group) = tile.scales[i];
            if (lane) return;
            const uint64_t at = tile.first_group * kGroup;
            const uint32_t n = tile.whole * kGroup;
            pipe::bulk_store(t.theta + at, sm.bytes[s] + F::kT, 2 * n);
            if (F::kRestBytes) pipe::bulk_store(static_cast<char*>(t.rest) + at * F::kRestBytes, sm.bytes[s] + F::kR, F::kRestBytes * n);
            pipe::bulk_store(static_cast<char*>(t.m) + at * F::kStateBytes, sm.bytes[s] + F::kM, F::kStateBytes * n);
            pipe::bulk_store(static_cast<char*>(t.v) + at * F::kStateBytes, sm.bytes[s] + F::kV, F::kStateBytes * n);
            pipe::bulk_commit();
        };
        AdamChunk next = blockIdx.x < a.num_tiles ? a.tiles[blockIdx.x] : AdamChunk{0, 0};
        for (uint64_t c = blockIdx.x; c < a.num_tiles; c += gridDim.x, ++it) {
            const uint32_t s = it % kStages;
            const AdamChunk chunk = next;
            if (c + gridDim.x < a.num_tiles) next = a.tiles[c + gridDim.x];
            const AdamRec& t = a.tensors[chunk.tensor];
            const uint64_t first_group = static_cast<uint64_t>(chunk.index) * kWarps, left = t.n - first_group * kGroup;
            const uint32_t groups = static_cast<uint32_t>(min((left + kGroup - 1) / kGroup, static_cast<uint64_t>(kWarps)));
            const uint32_t whole = t.aligned ? static_cast<uint32_t>(min(left / kGroup, static_cast<uint64_t>(kWarps))) : 0;
            if (it >= kStages) {
                alive = __all_sync(0xFFFFFFFFu, pipe::mbar_wait(&sm.done[s], (it / kStages - 1) & 1u, 300u + s, &g_adam_fault));
                if (!alive) break;
                store_out(s);
                if (lane == 0) pipe::bulk_wait_read_all();
                __syncwarp();
            }
            const uint64_t at = first_group * kGroup;
            const uint32_t n = whole * kGroup;
            if (STATE == COLLAGE_STATE_E4M3) {
                for (uint32_t i = lane; i < 2 * kWarps; i += 32)
                    if (i % kWarps < whole)
                        asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(pipe::smem_addr(&sm.tile[s].scales[i])), "l"(scale_at(t, i, first_group)) : "memory");
                asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(pipe::smem_addr(&sm.full[s])) : "memory");
            }
            if (lane == 0) {
                auto& tile = sm.tile[s];
                tile.tensor = &t;
                tile.first_group = first_group;
                tile.groups = groups;
                tile.whole = whole;
                // (a group's pairs begin at a multiple of 128: the lower word of their numbers passes 2^32 between groups only)
                const uint64_t pair = (t.first + at) >> 1;
                const uint32_t low = static_cast<uint32_t>(pair), high = static_cast<uint32_t>(pair >> 32);
                tile.random[0] = low + mix32(high + a.k.key);
                tile.random[1] = low + mix32(high + 1 + a.k.key);
                tile.passed = low ? (0u - low) / (kGroup / 2) : kWarps;
                pipe::mbar_arrive_expect_tx(&sm.full[s], n * (2 + (F::kReadsTheta ? 2 : 0) + F::kRestBytes + 2 * F::kStateBytes));
                if (n) {
                    pipe::bulk_load(sm.bytes[s] + F::kG, t.grad + at, 2 * n, &sm.full[s]);
                    if (F::kReadsTheta) pipe::bulk_load(sm.bytes[s] + F::kT, t.theta + at, 2 * n, &sm.full[s]);
                    if (F::kRestBytes) pipe::bulk_load(sm.bytes[s] + F::kR, static_cast<const char*>(t.rest) + at * F::kRestBytes, F::kRestBytes * n, &sm.full[s]);
                    pipe::bulk_load(sm.bytes[s] + F::kM, static_cast<const char*>(t.m) + at * F::kStateBytes, F::kStateBytes * n, &sm.full[s]);
                    pipe::bulk_load(sm.bytes[s] + F::kV, static_cast<const char*>(t.v) + at * F::kStateBytes, F::kStateBytes * n, &sm.full[s]);
                }
            }
        }
        for (uint32_t j = it > kStages ? it - kStages : 0; j < it && alive; ++j) {
            const uint32_t s = j % kStages;
            alive = __all_sync(0xFFFFFFFFu, pipe::mbar_wait(&sm.done[s], (j / kStages) & 1u, 310u + s, &g_adam_fault));
            if (alive) store_out(s);
        }
        // after a wait that was given up: the copies that are still under way
        for (uint32_t j = it > kStages ? it - kStages : 0; j < it && !alive; ++j)
            pipe::mbar_wait(&sm.full[j % kStages], (j / kStages) & 1u, 320u + j % kStages, &g_adam_fault);
        if (lane == 0) pipe::bulk_wait_all();
        return;
    }
    // Every warp takes part in every tile, so none can be a turn of a stage ahead of or behind its barriers.
    const float grad_scale = a.grad_scale ? *a.grad_scale : 1.0f;
    uint32_t s = 0, phase = 0;
    for (uint64_t c = blockIdx.x; c < a.num_tiles; c += gridDim.x) {
        if (!__all_sync(0xFFFFFFFFu, pipe::mbar_wait(&sm.full[s], phase, 330u + s, &g_adam_fault))) return;
        auto& tile = sm.tile[s];
        if (warp < tile.whole) {
            whole_group<STATE, REST, INSIDE>(sm.bytes[s], tile, warp, a.k, grad_scale, lane);
            pipe::fence_async_smem();
        } else if (warp < tile.groups) {
            any_group<STATE, REST, INSIDE>(*tile.tensor, tile.first_group + warp, a.k, grad_scale);
        }
        __syncwarp();
        if (lane == 0) pipe::mbar_arrive(&sm.done[s]);
        if (++s == kStages) { s = 0; phase ^= 1; }
    }
}

template <int STATE, int REST>
static collage_status_t launch_adam(const AdamArgs& a, int sm_count, cudaStream_t s) {
    const uint64_t grid = std::min<uint64_t>(a.num_tiles, sm_count);
    constexpr int threads = Form<STATE, REST>::kWarps * 32 + 32;
    if constexpr (STATE == COLLAGE_STATE_E4M3 || REST == COLLAGE_REST_BF16)          // (elsewhere the flat step's operations look at the flag)
        if (a.k.f.flags & COLLAGE_FLAG_EPS_INSIDE_SQRT)
            return launch<&adam_step_kernel<STATE, REST, true>>(grid, threads, 1, sizeof(AdamSmem<STATE, REST>), s, a);
    return launch<&adam_step_kernel<STATE, REST, false>>(grid, threads, 1, sizeof(AdamSmem<STATE, REST>), s, a);
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
    struct Part {                              // of a chunk: what is left of the tensor from its beginning on
        const uint16_t* grad;
        uint64_t left;
        bool aligned;
    };
    auto part_of = [&](uint64_t c) {
        if (c >= a.num_chunks) return Part{nullptr, 0, false};
        const AdamChunk chunk = a.chunks[c];
        const AdamRec& t = a.tensors[chunk.tensor];
        const uint64_t begin = chunk.index * static_cast<uint64_t>(kNormChunk);
        return Part{t.grad + begin, t.n - begin, t.aligned != 0};
    };
    Part now = part_of(blockIdx.x);
    for (uint64_t c = blockIdx.x; c < a.num_chunks; c += gridDim.x) {
        float g[2][8];
        uint4 q[2];
        const bool whole = now.aligned && now.left >= kNormChunk;
        if (whole) {
            q[0] = __ldcs(reinterpret_cast<const uint4*>(now.grad) + threadIdx.x);
            q[1] = __ldcs(reinterpret_cast<const uint4*>(now.grad) + threadIdx.x + kAdamThreads);
        }
        const Part next = part_of(c + gridDim.x);        // (looked up while the values are under way)
        if (whole) {
            unpack8(q[0], g[0]);
            unpack8(q[1], g[1]);
        } else {
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint32_t j = (i * 8 + e) * kAdamThreads + threadIdx.x;
                    g[i][e] = j < now.left ? bf16_value(now.grad[j]) : 0.0f;
                }
        }
        sum += squares(g[0]);
        sum += squares(g[1]);
        now = next;
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
    AdamChunk *d_chunks = nullptr, *d_tiles = nullptr;       // turns of the norm, and of the step
    uint64_t num_chunks = 0, num_tiles = 0;
    std::vector<ByteRange> ranges, written;    // sorted by address: all arrays, and those that a step writes
    int state = 0, rest = 0, device = -1;
    ~collage_adam_plan() {
        cudaFree(d_tensors);
        cudaFree(d_chunks);
        cudaFree(d_tiles);
    }
};

namespace {

collage_status_t create(const collage_adam_tensor_t* tensors, int num, int state, int rest, collage_adam_plan** out) {
    const uint64_t state_bytes = state == COLLAGE_STATE_F32 ? 4 : 1, rest_bytes = rest == COLLAGE_REST_F32 ? 4 : 2;
    std::vector<ByteRange> ranges, written;
    std::vector<AdamRec> recs;
    std::vector<AdamChunk> chunks, tiles;
    const uint32_t tile = tile_groups(rest);
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
        const uint64_t groups = (t.n + kGroup - 1) / kGroup, own_chunks = (t.n + kNormChunk - 1) / kNormChunk, own_tiles = (groups + tile - 1) / tile;
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
        r.aligned = !off(t.theta, 16) && !off(t.grad, 16) && !off(t.rest, 16) && !off(t.m, 16) && !off(t.v, 16);
        first += groups * kGroup;
        for (uint64_t c = 0; c < own_tiles; ++c) tiles.push_back({static_cast<uint32_t>(recs.size()), static_cast<uint32_t>(c)});
        for (uint64_t c = 0; c < own_chunks; ++c) chunks.push_back({static_cast<uint32_t>(recs.size()), static_cast<uint32_t>(c)});
        recs.push_back(r);
    }
    if (any_overlap(ranges)) return COLLAGE_ERR_ALIAS;
    any_overlap(written);                      // (sorts)
    DeviceInfo dev;
    if (const collage_status_t st = current_device(&dev); st != COLLAGE_OK) return st;
    collage_adam_plan* plan = new collage_adam_plan;
    plan->num_chunks = num_chunks;
    plan->num_tiles = tiles.size();
    plan->ranges = std::move(ranges);
    plan->written = std::move(written);
    plan->state = state;
    plan->rest = rest;
    if (cudaGetDevice(&plan->device) != cudaSuccess ||
        (num_chunks && (cudaMalloc(&plan->d_tensors, recs.size() * sizeof(AdamRec)) != cudaSuccess ||
                        cudaMalloc(&plan->d_chunks, chunks.size() * sizeof(AdamChunk)) != cudaSuccess ||
                        cudaMalloc(&plan->d_tiles, tiles.size() * sizeof(AdamChunk)) != cudaSuccess ||
                        cudaMemcpy(plan->d_tiles, tiles.data(), tiles.size() * sizeof(AdamChunk), cudaMemcpyHostToDevice) != cudaSuccess ||
                        cudaMemcpy(plan->d_tensors, recs.data(), recs.size() * sizeof(AdamRec), cudaMemcpyHostToDevice) != cudaSuccess ||
                        cudaMemcpy(plan->d_chunks, chunks.data(), chunks.size() * sizeof(AdamChunk), cudaMemcpyHostToDevice) != cudaSuccess ||
                        tables_landed() != cudaSuccess))) {
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

namespace collage {
cudaError_t read_clear_adam_fault(unsigned int* out) {
    unsigned int zero = 0;
    cudaError_t e = cudaMemcpyFromSymbol(out, g_adam_fault, sizeof *out);
    if (e == cudaSuccess && *out) e = cudaMemcpyToSymbol(g_adam_fault, &zero, sizeof zero);
    return e;
}
}  // namespace collage

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
    if (plan->num_tiles == 0) return COLLAGE_OK;
    AdamArgs a = {};
    a.tensors = plan->d_tensors;
    a.tiles = plan->d_tiles;
    a.num_tiles = plan->num_tiles;
    a.grad_scale = grad_scale;
    a.k.f = fp32_scalars(hyper, step);
    const double t = static_cast<double>(step), bc1 = 1.0 - std::pow(hyper->beta1, t), bc2 = 1.0 - std::pow(hyper->beta2, t);
    a.k.inv_bc1 = static_cast<float>(1.0 / bc1);
    a.k.rate = static_cast<float>(-hyper->lr / bc1);
    a.k.decay = static_cast<float>(-hyper->lr * hyper->weight_decay);
    a.k.a_hi = static_cast<float>(hyper->lr);
    a.k.a_lo = static_cast<float>(hyper->lr - a.k.a_hi);
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

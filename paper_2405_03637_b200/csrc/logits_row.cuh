// Rows of logits, shared by the losses that read them: 16-byte vectors of bfloat16 or float as pairs of floats, exponentials
// relative to a row's largest logit, rows that begin anywhere.
#pragma once
#include "ops_common.cuh"

namespace collage {
namespace ops {

constexpr float kLog2e = 1.4426950408889634f;

template <typename T>
struct Vec;                      // 16 bytes of logits, as kPairs pairs of floats
template <>
struct Vec<uint16_t> {
    static constexpr uint32_t kN = 8, kPairs = 4;
    static constexpr uint32_t kLowest = 0xFF80FF80u;          // minus infinity
    static __device__ __forceinline__ void unpack(const uint4& q, uint64_t (&f)[4]) {
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = pair_of(bf16_lo(w[i]), bf16_hi(w[i]));
    }
    static __device__ __forceinline__ uint4 pack(const uint64_t (&f)[4]) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 v = floats_of(f[i]);
            w[i] = pack_bf16(v.x, v.y);
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    // the largest so far, kept as it is stored (two running maxima); a NaN is passed over
    using Most = uint32_t;
    static __device__ __forceinline__ Most lowest() { return kLowest; }
    static __device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
        uint32_t r;
        asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        return r;
    }
    static __device__ __forceinline__ Most most(Most m, const uint4& q) { return max2(max2(max2(q.x, q.y), max2(q.z, q.w)), m); }
    static __device__ __forceinline__ float most_value(Most m) { return fmaxf(bf16_lo(m), bf16_hi(m)); }
    static __device__ __forceinline__ float value(uint16_t v) { return bf16_value(v); }
    static __device__ __forceinline__ uint16_t rounded(float v) { return to_bf16(v); }
};
template <>
struct Vec<float> {
    static constexpr uint32_t kN = 4, kPairs = 2;
    static constexpr uint32_t kLowest = 0xFF800000u;
    static __device__ __forceinline__ void unpack(const uint4& q, uint64_t (&f)[2]) {
        f[0] = pair_of(__uint_as_float(q.x), __uint_as_float(q.y));
        f[1] = pair_of(__uint_as_float(q.z), __uint_as_float(q.w));
    }
    static __device__ __forceinline__ uint4 pack(const uint64_t (&f)[2]) {
        const float2 a = floats_of(f[0]), b = floats_of(f[1]);
        return make_uint4(__float_as_uint(a.x), __float_as_uint(a.y), __float_as_uint(b.x), __float_as_uint(b.y));
    }
    using Most = float;
    static __device__ __forceinline__ Most lowest() { return -INFINITY; }
    static __device__ __forceinline__ Most most(Most m, const uint4& q) {
        return fmaxf(fmaxf(fmaxf(__uint_as_float(q.x), __uint_as_float(q.y)), fmaxf(__uint_as_float(q.z), __uint_as_float(q.w))), m);
    }
    static __device__ __forceinline__ float most_value(Most m) { return m; }
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

// exp2((f - m) c) of two logits.  The difference is taken first: z c - m c, an fma, would be rounded at the size of m c, however
// close z is to m.  `minus_m2` and `c2` are pairs of -m and c.
__device__ __forceinline__ float2 exps(uint64_t f, uint64_t minus_m2, uint64_t c2) {
    const float2 x = floats_of(mul_pair(add_pair(f, minus_m2), c2));
    return make_float2(fast_exp2(x.x), fast_exp2(x.y));
}
// exp2(f c - base) of two logits
__device__ __forceinline__ float2 based_exps(uint64_t f, uint64_t minus_base2, uint64_t c2) {
    const float2 x = floats_of(fma_pair(f, c2, minus_base2));
    return make_float2(fast_exp2(x.x), fast_exp2(x.y));
}
// Adds exp2((f - m) c) over a vector to `total`, or exp2(f c - RN(m c)) if BASED.  While there is no number yet (m = -infinity) every f is
// -infinity or NaN, and is taken as it is.
template <typename T, bool BASED>
__device__ __forceinline__ void add_exps(const uint4& q, float m, float c, uint64_t& total) {
    uint64_t f[Vec<T>::kPairs];
    Vec<T>::unpack(q, f);
    const float minus_m = m == -INFINITY ? 0.0f : -m;
#pragma unroll
    for (uint32_t i = 0; i < Vec<T>::kPairs; ++i) {
        const float2 e = BASED ? based_exps(f[i], pair_of(-m * c, -m * c), pair_of(c, c)) : exps(f[i], pair_of(minus_m, minus_m), pair_of(c, c));
        total = add_pair(total, pair_of(e.x, e.y));
    }
}

// Waits until at most `groups` of this thread's copy groups are under way (or 7, where more may be).
__device__ __forceinline__ void wait_pending(uint32_t groups) {
    switch (groups) {
        case 0: asm volatile("cp.async.wait_group 0;" ::: "memory"); break;
        case 1: asm volatile("cp.async.wait_group 1;" ::: "memory"); break;
        case 2: asm volatile("cp.async.wait_group 2;" ::: "memory"); break;
        case 3: asm volatile("cp.async.wait_group 3;" ::: "memory"); break;
        case 4: asm volatile("cp.async.wait_group 4;" ::: "memory"); break;
        case 5: asm volatile("cp.async.wait_group 5;" ::: "memory"); break;
        case 6: asm volatile("cp.async.wait_group 6;" ::: "memory"); break;
        default: asm volatile("cp.async.wait_group 7;" ::: "memory"); break;
    }
}

// A row as 16-byte vectors of its memory: vector v holds elements v kN - off ... of the row, those outside it do not exist.
template <typename T>
struct RowVectors {
    static constexpr uint32_t kN = Vec<T>::kN;
    uint4* base;                       // the row's first byte rounded down to 16
    T* row;
    uint32_t off, vocab;
    __device__ __forceinline__ RowVectors(T* r, uint32_t n) : row(r), vocab(n) {
        const uintptr_t a = reinterpret_cast<uintptr_t>(r);
        base = reinterpret_cast<uint4*>(a & ~static_cast<uintptr_t>(15));
        off = static_cast<uint32_t>(a & 15) / sizeof(T);
    }
    __device__ __forceinline__ uint32_t count() const { return (off + vocab + kN - 1) / kN; }
    __device__ __forceinline__ bool inside(uint32_t v) const { return (v || !off) && (v + 1) * kN <= off + vocab; }
    // vectors [whole_begin, whole_end) of the row lie inside it; at most one before and one behind them do not
    __device__ __forceinline__ uint32_t whole_begin() const { return off ? 1 : 0; }
    __device__ __forceinline__ uint32_t whole_end() const { return (off + vocab) / kN; }
    // a vector at the row's edge, missing elements as minus infinity
    __device__ __forceinline__ uint4 edge(uint32_t v) const {
        union { uint4 q; uint32_t w[4]; T e[kN]; } u;
        u.q = make_uint4(Vec<T>::kLowest, Vec<T>::kLowest, Vec<T>::kLowest, Vec<T>::kLowest);
#pragma unroll
        for (uint32_t i = 0; i < kN; ++i) {
            const int64_t e = static_cast<int64_t>(v) * kN + i - off;
            if (e >= 0 && e < vocab) u.e[i] = row[e];
        }
        return u.q;
    }
};

}  // namespace ops
}  // namespace collage

// Distillation from a teacher's top logits: loss, its gradient, and both in one pass.
//
// With z = logits / t and lse = log sum_j exp(z_j) over the vocabulary, the teacher's p over its own entries:
//   loss = t^2 sum_k p_k (log p_k - z_index(k) + lse),   dlogits_j = g t (exp(z_j - lse) - sum_{index(k) = j} p_k).
// Both softmaxes are taken on differences from the row's largest logit m, before the division by t: a row whose logits all
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
    float inv_t_rest;           // what inv_t lacks of 1 / t
};

constexpr uint32_t kSeenWords = 256;           // bitmaps over the indexes of a row, modulo 2^13
constexpr uint32_t kMaxCluster = 8;
constexpr float kLog2e = 1.4426950408889634f;
// A stored lse of this size or more is rounded too coarsely to give q to 2^-17 (an infinite one to give it at all): the
// backward pass then takes maximum and sum from the row again.
constexpr float kLargeLse = 128.0f;
constexpr size_t kSmSmem = 228 * 1024, kMaxSmem = 227 * 1024 - 5 * 1024;   // of an SM; dynamic part that a block may take
constexpr size_t kThird = 74 * 1024 - 4608, kHalf = 112 * 1024 - 4608;     // dynamic parts of a third and of half an SM

// Two floats in a 64-bit register: one instruction works on both.
__device__ __forceinline__ uint64_t pair_of(float lo, float hi) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ float2 floats_of(uint64_t v) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
    return r;
}
__device__ __forceinline__ uint64_t fma_pair(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t add_pair(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t mul_pair(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

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

// exp((x - most) / t), and the exponent rounded to `shifted`.  Its roundings (of the difference, of 1 / t and of their product)
// are followed up: in the loss an entry's p may be multiplied by a -log q of any size.
__device__ __forceinline__ float teacher_exp(float x, float most, const DistillArgs& a, float& shifted) {
    const float d = x - most, back = x - d, rest = (x - (d + back)) + (back - most);
    shifted = d * a.inv_t;
    const float lost = __fmaf_rn(d, a.inv_t, -shifted) + __fmaf_rn(rest, a.inv_t, d * a.inv_t_rest), e = expf(shifted);
    return shifted > -128.0f ? __fmaf_rn(e, lost, e) : e;             // (below, e is 0 and what is lost may be infinite; a NaN passes)
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
// Staged bfloat16 rows, which instructions bound, take the fma all the same, with RN(m c) as the base, as long as what that lacks of m c
// (lack(), exact) is a quarter at most: every exponential is off by the factor exp2(lack) then, and sums are divided by it.
// (4096 x 32000: 105 us, 115 by differences; in float 219 us by differences, 234 by the fma.)
constexpr float kLargeShift = 0x1p22f;
template <typename T>
__device__ __forceinline__ bool by_base(float m, float c) { return sizeof(T) == 2 && fabsf(m * c) < kLargeShift; }
template <typename T>
__device__ __forceinline__ float lack(float m, float c) { return by_base<T>(m, c) ? __fmaf_rn(m, c, -(m * c)) : 0.0f; }

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

// What a row's blocks share, apart from the row itself.
struct DistillShared {
    float2 warp[8];
    float2 part[kMaxCluster];          // (maximum, sum) of each block of the cluster
    float loss[kMaxCluster];
    int any_there;
    float log_psum;
};

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

// A row of `vocab` logits by a cluster of blocks, each with a slice of it that it streams from global memory, once for
// maximum and sum and once for the gradient.  MODE 0: loss (and lse).  1: gradient from a stored lse.  2: both (rows
// that are too long to be staged).
template <typename T, int MODE, int kDistillThreads>
__global__ void __launch_bounds__(kDistillThreads, (MODE == 0 ? 2048 : 1280) / kDistillThreads) distill_kernel(const __grid_constant__ DistillArgs a) {
    using V = Vec<T>;
    constexpr uint32_t kN = V::kN;
    extern __shared__ __align__(16) uint8_t dynamic[];
    __shared__ DistillShared sh;
    after_previous();
    float* tp = reinterpret_cast<float*>(dynamic);              // teacher: p, student's logit, index
    float* tz = tp + a.k;
    int* ti = reinterpret_cast<int*>(tz + a.k);
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = a.cluster > 1 ? umma::cluster_rank() : 0;
    const uint64_t row = blockIdx.x / a.cluster;
    const RowVectors<T> z(const_cast<T*>(static_cast<const T*>(a.logits)) + row * a.ldz, a.vocab);
    const RowVectors<T> dz(MODE ? static_cast<T*>(a.dlogits) + row * a.ldd : nullptr, a.vocab);
    const uint32_t first = rank * a.slice, end = min(first + a.slice, z.count());        // this block's vectors
    const float g = MODE ? a.row_scale[row] : 1.0f;

    constexpr uint32_t kAhead = 4;              // vectors in flight for a thread
    const uint4 lowest = make_uint4(V::kLowest, V::kLowest, V::kLowest, V::kLowest);
    // Whole vectors of the slice; the row's first and last one may be cut.
    const uint32_t whole = first + (first < end && !z.inside(first)), whole_end = max(whole, end - (first < end && !z.inside(end - 1)));
    // Gradients of the slice: `load(v)` gives a whole vector of logits, `element(e)` one of them, `value` turns a pair of
    // logits into gradients.  Cut vectors, and rows whose gradients lie otherwise in their vectors, go by elements.
    auto write_row = [&](auto&& load, auto&& element, auto&& value) {
        auto by_elements = [&](uint32_t lo, uint32_t hi) {
#pragma unroll 1
            for (uint32_t e = lo + threadIdx.x; e < hi; e += kDistillThreads) dz.row[e] = V::rounded(floats_of(value(pair_of(element(e), 0.0f))).x);
        };
        const uint32_t lo = first ? first * kN - z.off : 0, hi = min(end * kN - z.off, a.vocab);
        if (z.off != dz.off) return by_elements(lo, hi);
        auto put = [&](uint32_t v, const uint4& q) {
            uint64_t f[V::kPairs];
            V::unpack(q, f);
#pragma unroll
            for (uint32_t i = 0; i < V::kPairs; ++i) f[i] = value(f[i]);
            dz.base[v] = V::pack(f);
        };
        uint32_t v = whole + threadIdx.x;
        for (; v + (kAhead - 1) * kDistillThreads < whole_end; v += kDistillThreads * kAhead) {
            uint4 q[kAhead];
#pragma unroll
            for (uint32_t i = 0; i < kAhead; ++i) q[i] = load(v + i * kDistillThreads);
#pragma unroll
            for (uint32_t i = 0; i < kAhead; ++i) put(v + i * kDistillThreads, q[i]);
        }
#pragma unroll 1
        for (; v < whole_end; v += kDistillThreads) put(v, load(v));
        if (whole > first) by_elements(lo, min(whole * kN - z.off, hi));
        if (whole_end < end) by_elements(whole_end * kN - z.off, hi);
    };
    auto zeros = [&] {
        write_row([&](uint32_t) { return lowest; }, [](uint32_t) { return 0.0f; }, [](uint64_t) -> uint64_t { return 0; });
    };
    if (MODE && g == 0.0f) {
        zeros();
        if (MODE == 2 && rank == 0 && threadIdx.x == 0) a.loss[row] = 0.0f;
        return;
    }
    if (a.cluster > 1) umma::cluster_arrive_all();                       // this block runs
    auto vector = [&](uint32_t v) { return z.base[v]; };
    auto element = [&](uint32_t e) { return V::value(z.row[e]); };

    if (warp == 0) {                            // the teacher's entries: p over all of them, in every block of the row
        float most = -INFINITY;
        bool bad = false;
        for (uint32_t k = lane; k < a.k; k += 32) {
            const uint64_t at = row * a.ldi + k;
            const int64_t i = a.index_bytes == 8 ? static_cast<const int64_t*>(a.top_index)[at] : static_cast<const int32_t*>(a.top_index)[at];
            const bool there = i >= 0 && i < static_cast<int64_t>(a.vocab);
            const float t = there ? a.top_logits[row * a.ldt + k] : -INFINITY;
            ti[k] = there ? static_cast<int>(i) : -1;
            tp[k] = t;
            most = fmaxf(most, t);
            bad |= t != t;
        }
        most = warp_max(most);
        const bool any_there = __any_sync(0xFFFFFFFFu, bad) || most > -INFINITY;
        float psum = 0.0f;
        for (uint32_t k = lane; k < a.k; k += 32) {
            tp[k] = teacher_exp(tp[k], most, a, tz[k]);      // (tz: until the student's logit takes its place)
            psum += tp[k];
        }
        psum = warp_sum(psum);
        for (uint32_t k = lane; k < a.k; k += 32) tp[k] /= psum;
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
        uint64_t total = 0;
        auto take = [&](const uint4 (&q)[kAhead]) {
            typename V::Most most = V::lowest();
#pragma unroll
            for (uint32_t i = 0; i < kAhead; ++i) most = V::most(most, q[i]);
            const float to = fmaxf(m, V::most_value(most));
            if (to != m) {                  // a new maximum: what is summed so far is taken relative to it
                const float2 so_far = floats_of(total);
                total = pair_of(rescaled(so_far.x, m, to, c), rescaled(so_far.y, m, to, c));
                m = to;
            }
#pragma unroll
            for (uint32_t i = 0; i < kAhead; ++i) add_exps<T, false>(q[i], m, c, total);
        };
        for (uint32_t v = whole + threadIdx.x; v < whole_end; v += kDistillThreads * kAhead) {
            uint4 q[kAhead];
#pragma unroll
            for (uint32_t i = 0; i < kAhead; ++i) q[i] = v + i * kDistillThreads < whole_end ? z.base[v + i * kDistillThreads] : lowest;
            take(q);
        }
        if (threadIdx.x ? threadIdx.x == 1 && whole_end < end : whole > first) {       // cut vectors: one thread for each
            uint4 q[kAhead] = {z.edge(threadIdx.x ? end - 1 : first), lowest, lowest, lowest};
            take(q);
        }
        const float2 sums = floats_of(total);
        sum = sums.x + sums.y;
        float most = warp_max(m);
        sum = warp_sum(rescaled(sum, m, most, c));
        if (lane == 0) sh.warp[warp] = make_float2(most, sum);
        __syncthreads();
        const float2 w = lane < kDistillThreads / 32 ? sh.warp[lane] : make_float2(-INFINITY, 0.0f);
        m = warp_max(w.x);
        sum = warp_sum(rescaled(w.y, w.x, m, c));
        if (a.cluster > 1) {
            umma::cluster_wait_all();           // all blocks of the row run
            if (threadIdx.x < a.cluster) {
                const uint32_t to = umma::cluster_addr(&sh.part[rank], threadIdx.x);
                asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(to), "f"(m), "f"(sum) : "memory");
            }
            umma::cluster_sync_any();
            const float2 r = lane < a.cluster ? sh.part[lane] : make_float2(-INFINITY, 0.0f);
            m = warp_max(r.x);
            sum = warp_sum(rescaled(r.y, r.x, m, c));
        }
    } else {
        __syncthreads();
        if (a.cluster > 1) umma::cluster_wait_all();
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
    // q_j = exp2((z_j - m) c) / sum, or exp2(z_j c - log2sum) by a stored lse
    const bool stored = MODE == 1 && !from_row;
    const float log2sum = lse * kLog2e, scale = __fdividef(1.0f, sum);
    auto q_of = [&](float v) { return stored ? fast_exp2(__fmaf_rn(v, c, -log2sum)) : fast_exp2((v - m) * c) * scale; };

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
            const float v = V::value(z.row[i]);
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
        umma::cluster_sync_any();
        if (MODE != 1 && rank == 0 && threadIdx.x == 0) {
            float loss = 0.0f;
            for (uint32_t r = 0; r < a.cluster; ++r) loss += sh.loss[r];
            a.loss[row] = (MODE == 2 ? g : 1.0f) * (loss * a.t * a.t);
        }
    } else {
        __syncthreads();
    }
    if (MODE) {
        const float gt = g * a.t, gs = gt * scale;
        const uint64_t c2 = pair_of(c, c), g2 = pair_of(gs, gs);
        if (stored) {                           // (sum and scale are 1)
            const uint64_t s2 = pair_of(-log2sum, -log2sum);
            write_row(vector, element, [&](uint64_t f) {
                const float2 e = based_exps(f, s2, c2);
                return mul_pair(g2, pair_of(e.x, e.y));
            });
        } else {
            const uint64_t m2 = pair_of(-m, -m);
            write_row(vector, element, [&](uint64_t f) {
                const float2 e = exps(f, m2, c2);
                return mul_pair(g2, pair_of(e.x, e.y));
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

// Loss and gradient of rows that fit the shared memory of a cluster: each block keeps its slice of a row between the two
// passes over it and walks over rows.  A thread owns the same places of the slice for every row: as soon as it has made
// the gradient of a place it sends for the next row's vector, so loads, exponentials and stores of two rows overlap.
// One more warp has the teacher's entries: their softmax while the others sum, the student's logits at them before the
// places are overwritten, then the loss, and one row later, when the dense gradient is surely written, the entries over it.
struct StagedShared {
    float2 warp[12];
    float2 part[2][kMaxCluster];          // (maximum, sum) of each block of the cluster; two rows' worth, as all below
    float loss[2][kMaxCluster];
    uint32_t seen[2][kSeenWords], again[2][kSeenWords];
    int any_there[2];
    struct {                              // what is still to be done for the row before
        void* line;
        unsigned long long row;
        float m, scale, g;
        uint32_t off, end;
        int small, live;
    } last;
};

template <typename T, int kStagedThreads, int BLOCKS>
__global__ void __launch_bounds__(kStagedThreads + 32, BLOCKS) distill_staged_kernel(const __grid_constant__ DistillArgs a, uint64_t rows) {
    using V = Vec<T>;
    constexpr uint32_t kN = V::kN;
    extern __shared__ __align__(16) uint8_t dynamic[];
    __shared__ StagedShared sh;
    uint4* stage = reinterpret_cast<uint4*>(dynamic);                                     // [slice]
    int64_t* raw_index = reinterpret_cast<int64_t*>(dynamic + 16ull * a.slice);           // [k], 4 or 8 bytes each: as it came
    float* raw_top = reinterpret_cast<float*>(raw_index + a.k);                           // [k]
    float* all_p = raw_top + a.k;                                                         // [2][k] teacher's p
    float* all_z = all_p + 2 * a.k;                                                       // [2][k] student's logit
    int* all_i = reinterpret_cast<int*>(all_z + 2 * a.k);                                 // [2][k] index, -1 = absent
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const bool teacher = threadIdx.x >= kStagedThreads;
    const uint32_t rank = a.cluster > 1 ? umma::cluster_rank() : 0, first = rank * a.slice;
    const uint64_t step = gridDim.x / a.cluster;
    const float c = a.inv_t * kLog2e;
    const uint32_t stage_addr = umma::smem_addr(stage);
    after_previous();

    auto logits_of = [&](uint64_t row) { return RowVectors<T>(const_cast<T*>(static_cast<const T*>(a.logits)) + row * a.ldz, a.vocab); };
    auto send_for = [&](const RowVectors<T>& z, uint32_t v) {
        if (z.inside(v))
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(stage_addr + 16 * (v - first)), "l"(z.base + v) : "memory");
        else
            stage[v - first] = z.edge(v);
    };
    // A thread's places are taken in batches; its copies are counted by batch too, so that the first of a row can be used
    // while the last are under way.
    constexpr uint32_t kAhead = 4, kBatch = kAhead * kStagedThreads;
    auto batches = [&](uint32_t end) { return (end - min(first, end) + kBatch - 1) / kBatch; };
    auto send_for_teacher = [&](uint64_t row) {
        for (uint32_t k = lane; k < a.k; k += 32) {
            const uint64_t at = row * a.ldi + k;
            if (a.index_bytes == 8)
                asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(umma::smem_addr(raw_index + k)), "l"(static_cast<const int64_t*>(a.top_index) + at) : "memory");
            else
                asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(umma::smem_addr(reinterpret_cast<int32_t*>(raw_index) + k)), "l"(static_cast<const int32_t*>(a.top_index) + at) : "memory");
            asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(umma::smem_addr(raw_top + k)), "l"(a.top_logits + row * a.ldt + k) : "memory");
        }
    };

    uint64_t row = blockIdx.x / a.cluster;
    float g = row < rows ? a.row_scale[row] : 0.0f;
    if (a.cluster > 1) umma::cluster_sync_any();    // all blocks run before one writes into another
    if (g != 0.0f) {
        if (teacher) {
            send_for_teacher(row);
        } else {
            const RowVectors<T> z = logits_of(row);
            const uint32_t end = min(first + a.slice, z.count());
            for (uint32_t n = 0; n < batches(end); ++n) {
                for (uint32_t v = first + n * kBatch + threadIdx.x; v < min(first + (n + 1) * kBatch, end); v += kStagedThreads) send_for(z, v);
                asm volatile("cp.async.commit_group;" ::: "memory");
            }
        }
    }
    uint32_t turn = 0;                          // rows with a distribution so far
    auto inside = [&](int i, uint32_t off, uint32_t end) {              // is entry i in this block's slice?
        const uint32_t v = (static_cast<uint32_t>(i) + off) / kN;
        return i >= 0 && v >= first && v < end;
    };
    auto finish_last = [&](uint32_t b) {        // the teacher's warp, for the row before; b: its buffers
        const auto& last = sh.last;
        if (a.cluster > 1 && rank == 0 && lane == 0) {
            float loss = 0.0f;
            for (uint32_t r = 0; r < a.cluster; ++r) loss += sh.loss[b][r];
            a.loss[last.row] = last.live ? last.g * (loss * a.t * a.t) : 0.0f;
        }
        if (!last.live) return;
        const float *tp = all_p + b * a.k, *tz = all_z + b * a.k;
        const int* ti = all_i + b * a.k;
        for (uint32_t k = lane; k < a.k; k += 32) {
            const int i = ti[k];
            if (!inside(i, last.off, last.end)) continue;
            float p = tp[k];
            // an index that appears more than once: all its lanes add up the same sum.  (Indexes that share a bit are searched
            // too, and found alone.)
            if (sh.again[b][(static_cast<uint32_t>(i) >> 5) % kSeenWords] >> (i & 31) & 1) {
                p = 0.0f;
                for (uint32_t o = 0; o < a.k; ++o)
                    if (ti[o] == i) p += tp[o];
            }
            const float x = last.small ? __fmaf_rn(tz[k], c, -last.m * c) : (tz[k] - last.m) * c;
            static_cast<T*>(last.line)[i] = V::rounded(last.g * a.t * (fast_exp2(x) * last.scale - p));
        }
    };

    for (; row < rows; row += step) {
        const RowVectors<T> z = logits_of(row), dz(static_cast<T*>(a.dlogits) + row * a.ldd, a.vocab);
        const uint32_t end = min(first + a.slice, z.count());
        const bool more = row + step < rows;
        const float g_next = more ? a.row_scale[row + step] : 0.0f;
        const RowVectors<T> zn = logits_of(more ? row + step : row);
        const uint32_t end_next = g_next != 0.0f ? min(first + a.slice, zn.count()) : 0;

        const uint32_t next_batches = batches(end_next);
        // Gradients of this thread's places, and the next row into them.  `value(f)` puts gradients in the logits' place.
        const bool alike = z.off == dz.off;
        // batches of places that are whole vectors of both rows need no further checks
        const uint32_t plain_begin = max(z.whole_begin(), end_next ? zn.whole_begin() : 0);
        const uint32_t plain_end = alike ? min(min(z.whole_end(), end), end_next ? min(zn.whole_end(), end_next) : end) : 0;
        auto write_row = [&](bool staged, auto&& value) {
            const uint32_t stop = max(end, end_next);
            uint32_t n_batch = 0;
#pragma unroll 1
            for (uint32_t begin = first; begin < stop; begin += kBatch, ++n_batch) {
                const uint32_t v0 = begin + threadIdx.x;
                if (v0 >= plain_begin && v0 + (kBatch - kStagedThreads) < plain_end) {
                    uint64_t f[kAhead][V::kPairs];
                    if (staged) {
#pragma unroll
                        for (uint32_t n = 0; n < kAhead; ++n) V::unpack(stage[v0 - first + n * kStagedThreads], f[n]);
                    }
#pragma unroll
                    for (uint32_t n = 0; n < kAhead; ++n) value(f[n]);
                    if (end_next) {
#pragma unroll
                        for (uint32_t n = 0; n < kAhead; ++n)
                            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(stage_addr + 16 * (v0 - first + n * kStagedThreads)),
                                         "l"(zn.base + v0 + n * kStagedThreads)
                                         : "memory");
                    }
#pragma unroll
                    for (uint32_t n = 0; n < kAhead; ++n) dz.base[v0 + n * kStagedThreads] = V::pack(f[n]);
                } else {
#pragma unroll 1
                    for (uint32_t v = v0; v < min(v0 + kBatch, stop); v += kStagedThreads) {
                        uint64_t f[V::kPairs];
                        V::unpack(stage[v - first], f);
                        value(f);
                        if (v < end_next) send_for(zn, v);
                        if (v >= end) continue;
                        if (alike && z.inside(v)) {
                            dz.base[v] = V::pack(f);
                        } else {
#pragma unroll
                            for (uint32_t i = 0; i < kN; ++i) {
                                const int64_t e = static_cast<int64_t>(v) * kN + i - z.off;
                                const float2 p = floats_of(f[i / 2]);
                                if (e >= 0 && e < a.vocab) dz.row[e] = V::rounded(i % 2 ? p.y : p.x);
                            }
                        }
                    }
                }
                if (n_batch < next_batches) asm volatile("cp.async.commit_group;" ::: "memory");
            }
        };
        auto zero = [](uint64_t (&f)[V::kPairs]) {
#pragma unroll
            for (uint32_t i = 0; i < V::kPairs; ++i) f[i] = 0;
        };
        if (g == 0.0f) {                        // weighs nothing: not read
            if (!teacher) {
                write_row(false, zero);
            } else {
                if (end_next) send_for_teacher(row + step);
                if (rank == 0 && lane == 0) a.loss[row] = 0.0f;
            }
            g = g_next;
            continue;
        }
        const uint32_t b = turn & 1;
        float *tp = all_p + b * a.k, *tz = all_z + b * a.k;
        int* ti = all_i + b * a.k;
        float log_psum = 0.0f, m = -INFINITY, sum = 0.0f;
        if (teacher) {
            asm volatile("cp.async.wait_all;" ::: "memory");
            __syncwarp();
            float most = -INFINITY, psum = 0.0f;
            bool bad = false;
            for (uint32_t k = lane; k < a.k; k += 32) {
                const int64_t i = a.index_bytes == 8 ? raw_index[k] : reinterpret_cast<const int32_t*>(raw_index)[k];
                const bool there = i >= 0 && i < static_cast<int64_t>(a.vocab);
                const float t = there ? raw_top[k] : -INFINITY;
                ti[k] = there ? static_cast<int>(i) : -1;
                tp[k] = t;
                most = fmaxf(most, t);
                bad |= t != t;
            }
            most = warp_max(most);
            const bool any_there = __any_sync(0xFFFFFFFFu, bad) || most > -INFINITY;
            for (uint32_t k = lane; k < a.k; k += 32) {
                tp[k] = teacher_exp(tp[k], most, a, tz[k]);  // (tz: until the student's logit takes its place)
                psum += tp[k];
            }
            psum = warp_sum(psum);
            log_psum = logf(psum);
            for (uint32_t k = lane; k < a.k; k += 32) tp[k] /= psum;
            if (lane == 0) sh.any_there[b] = any_there;
            for (uint32_t i = lane; i < kSeenWords; i += 32) sh.seen[b][i] = sh.again[b][i] = 0;
        } else {
            // Maximum (batch by batch as they come: a thread reads what it has sent for itself), then sum of this thread's vectors.
            const uint32_t mine = batches(end);
            auto each_place = [&](bool wait, auto&& f) {
#pragma unroll 1
                for (uint32_t n = 0; n < mine; ++n) {
                    if (wait) wait_pending(mine - 1 - n);
                    const uint32_t v0 = n * kBatch + threadIdx.x;
                    if ((n + 1) * kBatch <= end - first) {
                        uint4 q[kAhead];
#pragma unroll
                        for (uint32_t i = 0; i < kAhead; ++i) q[i] = stage[v0 + i * kStagedThreads];
#pragma unroll
                        for (uint32_t i = 0; i < kAhead; ++i) f(q[i], i);
                    } else {
#pragma unroll
                        for (uint32_t i = 0; i < kAhead; ++i)
                            if (v0 + i * kStagedThreads < end - first) f(stage[v0 + i * kStagedThreads], i);
                    }
                }
            };
            typename V::Most largest[2] = {V::lowest(), V::lowest()};
            each_place(true, [&](const uint4& q, uint32_t i) { largest[i & 1] = V::most(largest[i & 1], q); });
            m = fmaxf(V::most_value(largest[0]), V::most_value(largest[1]));
            uint64_t total[2] = {0, 0};
            if (by_base<T>(m, c))
                each_place(false, [&](const uint4& q, uint32_t i) { add_exps<T, true>(q, m, c, total[i & 1]); });
            else
                each_place(false, [&](const uint4& q, uint32_t i) { add_exps<T, false>(q, m, c, total[i & 1]); });
            const float2 sums = floats_of(add_pair(total[0], total[1]));
            sum = (sums.x + sums.y) * fast_exp2(-lack<T>(m, c));
            const float most = warp_max(m);
            sum = warp_sum(rescaled(sum, m, most, c));
            if (lane == 0) sh.warp[warp] = make_float2(most, sum);
        }
        __syncthreads();                        // all sums, the whole slice and the teacher's p are there; the last row's gradient is written
        const float2 w = lane < kStagedThreads / 32 ? sh.warp[lane] : make_float2(-INFINITY, 0.0f);
        m = warp_max(w.x);
        sum = warp_sum(rescaled(w.y, w.x, m, c));
        if (a.cluster > 1) {
            if (threadIdx.x < a.cluster) {
                const uint32_t to = umma::cluster_addr(&sh.part[b][rank], threadIdx.x);
                asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(to), "f"(m), "f"(sum) : "memory");
            }
            umma::cluster_sync_any();
            const float2 r = lane < a.cluster ? sh.part[b][lane] : make_float2(-INFINITY, 0.0f);
            m = warp_max(r.x);
            sum = warp_sum(rescaled(r.y, r.x, m, c));
        }
        if (m == -INFINITY) sum = NAN;          // a row without any number in it has no distribution
        const bool small = by_base<T>(m, c), live = sh.any_there[b];
        float loss = 0.0f;
        if (teacher) {                          // the student's logits at the entries in this block's slice, and their part of the loss
            const float logsum = logf(sum);
            for (uint32_t k = lane; k < a.k; k += 32) {
                const int i = ti[k];
                if (!inside(i, z.off, end)) continue;
                const float v = V::value(reinterpret_cast<const T*>(stage)[static_cast<uint32_t>(i) + z.off - first * kN]), p = tp[k];
                if (!(p == 0.0f)) loss = __fmaf_rn(p, tz[k] - log_psum - ((v - m) * a.inv_t - logsum), loss);
                tz[k] = v;
            }
        }
        __syncthreads();                        // the slice may be overwritten
        const float scale = __fdividef(fast_exp2(-lack<T>(m, c)), sum), gs = g * a.t * scale;           // turns exponentials into q, and into gradients
        if (teacher) {
            if (turn > 0) finish_last(b ^ 1);
            loss = warp_sum(loss);
            if (lane == 0) {
                if (a.cluster > 1)
                    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(umma::cluster_addr(&sh.loss[b][rank], 0)), "f"(loss) : "memory");
                else
                    a.loss[row] = live ? g * (loss * a.t * a.t) : 0.0f;
            }
            for (uint32_t k = lane; k < a.k; k += 32) {
                const int i = ti[k];
                if (!inside(i, z.off, end)) continue;
                const uint32_t bit = 1u << (i & 31), word = (static_cast<uint32_t>(i) >> 5) % kSeenWords;
                if (atomicOr(&sh.seen[b][word], bit) & bit) atomicOr(&sh.again[b][word], bit);
            }
            __syncwarp();
            if (end_next) send_for_teacher(row + step);
            __syncwarp();
            if (lane == 0) sh.last = {dz.row, row, m, scale, g, z.off, end, small, live};
            __syncwarp();
        } else if (!live) {                     // nothing to learn from: zeros whatever the logits are
            write_row(false, zero);
        } else if (small) {
            const uint64_t c2 = pair_of(c, c), b2 = pair_of(-m * c, -m * c), g2 = pair_of(gs, gs);
            write_row(true, [&](uint64_t (&f)[V::kPairs]) {
#pragma unroll
                for (uint32_t i = 0; i < V::kPairs; ++i) {
                    const float2 e = based_exps(f[i], b2, c2);
                    f[i] = mul_pair(g2, pair_of(e.x, e.y));
                }
            });
        } else {
            write_row(true, [&](uint64_t (&f)[V::kPairs]) {
#pragma unroll
                for (uint32_t i = 0; i < V::kPairs; ++i) {
                    if constexpr (sizeof(T) == 2) {     // (rare here, and in packed instructions it would cost the ordinary rows registers)
                        const float2 x = floats_of(f[i]);
                        f[i] = pair_of(gs * fast_exp2((x.x - m) * c), gs * fast_exp2((x.y - m) * c));
                    } else {
                        const float2 e = exps(f[i], pair_of(-m, -m), pair_of(c, c));
                        f[i] = mul_pair(pair_of(gs, gs), pair_of(e.x, e.y));
                    }
                }
            });
        }
        g = g_next;
        ++turn;
    }
    __syncthreads();                            // the last row's gradient is written
    if (a.cluster > 1) umma::cluster_sync_any();    // its losses have come; no block leaves while another may still write to it
    if (teacher && turn > 0) finish_last((turn - 1) & 1);
}

template <typename T, int THREADS, int BLOCKS>
static collage_status_t launch_staged_as(const DistillArgs& a, uint64_t rows, int sm_count, cudaStream_t s) {
    const size_t smem = 16ull * a.slice + 36ull * a.k;
    const uint64_t fit = std::max<uint64_t>(1, std::min<uint64_t>(BLOCKS, kSmSmem / (smem + sizeof(StagedShared) + 1024)));
    const uint64_t groups = std::min<uint64_t>(rows, std::max<uint64_t>(1, fit * sm_count / a.cluster));
    return launch<&distill_staged_kernel<T, THREADS, BLOCKS>>(groups * a.cluster, THREADS + 32, a.cluster, smem, s, a, rows);
}
// Threads by the slice's vectors: about twenty each of the longest; short rows by smaller blocks, more of them on an SM.  Rows of
// which only two fit an SM are still faster whole than halved over a cluster: 1306 x 100352 129 us against 173.
template <typename T>
static collage_status_t launch_staged(const DistillArgs& a, uint64_t rows, int sm_count, cudaStream_t s) {
    return a.slice <= 512    ? launch_staged_as<T, 64, 8>(a, rows, sm_count, s)
           : a.slice <= 1536 ? launch_staged_as<T, 128, 5>(a, rows, sm_count, s)
           : 16ull * a.slice + 36ull * a.k <= kThird ? launch_staged_as<T, 256, 3>(a, rows, sm_count, s)
                                                     : launch_staged_as<T, 384, 2>(a, rows, sm_count, s);
}

// Short rows by smaller blocks, more of them on an SM: 16384 x 4000 backward 82 us by 128 threads, 122 by 256; the loss 43 and 76.
template <typename T, int MODE>
static collage_status_t launch_streamed(const DistillArgs& a, uint64_t rows, cudaStream_t s) {
    const size_t smem = 12ull * a.k;
    if constexpr (MODE != 2) {                      // (that mode comes here with long rows only)
        if (a.slice <= 256) return launch<&distill_kernel<T, MODE, 64>>(rows * a.cluster, 64, a.cluster, smem, s, a);
        if (a.slice <= 1024) return launch<&distill_kernel<T, MODE, 128>>(rows * a.cluster, 128, a.cluster, smem, s, a);
    }
    return launch<&distill_kernel<T, MODE, 256>>(rows * a.cluster, 256, a.cluster, smem, s, a);
}

template <int MODE>
static collage_status_t launch_distill(DistillArgs& a, uint64_t rows, collage_dtype_t dtype, int sm_count, void* stream) {
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const bool bf16 = dtype == COLLAGE_DTYPE_BF16;
    const uint32_t per_vector = bf16 ? 8 : 4;
    const uint32_t vectors = (a.vocab + 2 * per_vector - 2) / per_vector;        // at the worst alignment
    a.cluster = 1;
    auto slice = [&] { return (vectors + a.cluster - 1) / a.cluster; };
    // few rows: more blocks for each, up to `per_sm` on an SM in all and down to `least` vectors each
    auto spread = [&](uint64_t per_sm, uint32_t least) {
        while (a.cluster < kMaxCluster && rows * a.cluster * 2 <= per_sm * sm_count && slice() >= 2 * least) a.cluster *= 2;
        a.slice = slice();
    };
    if constexpr (MODE == 2) {
        const size_t teacher = 36ull * a.k;
        // two or three blocks of an SM hold their slices; beyond eight of those, one block may take all of the shared memory
        while (a.cluster < kMaxCluster && 16ull * slice() + teacher > kHalf) a.cluster *= 2;
        if (16ull * slice() + teacher <= kMaxSmem) {
            spread(1, 256);
            return bf16 ? launch_staged<uint16_t>(a, rows, sm_count, s) : launch_staged<float>(a, rows, sm_count, s);
        }
        a.cluster = 1;
    }
    spread(4, 512);                      // (115 x 71270 float: loss 14 us, backward 17; 22 and 24 with one block for each SM)
    return bf16 ? launch_streamed<uint16_t, MODE>(a, rows, s) : launch_streamed<float, MODE>(a, rows, s);
}

// Everything the three entry points check alike; `read` and `written` are their float[rows] arrays.
static collage_status_t prepare_distill(const collage_distill_t* in, const float* const (&read)[2], float* const (&written)[2],
                                        const collage_matrix_t* dlogits, DistillArgs* out, DeviceInfo* dev) {
    const uint32_t size = in->logits_dtype == COLLAGE_DTYPE_BF16 ? 2 : 4;
    if (in->logits_dtype != COLLAGE_DTYPE_BF16 && in->logits_dtype != COLLAGE_DTYPE_F32) return COLLAGE_ERR_ARG;
    if (in->top_index_bytes != 4 && in->top_index_bytes != 8) return COLLAGE_ERR_ARG;
    if (!(std::isfinite(in->temperature) && in->temperature > 0.0)) return COLLAGE_ERR_ARG;
    const float t = static_cast<float>(in->temperature), inv_t = static_cast<float>(1.0 / in->temperature);
    if (!(t > 0.0f && std::isfinite(t) && inv_t > 0.0f && std::isfinite(inv_t * kLog2e))) return COLLAGE_ERR_ARG;
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
    out->inv_t_rest = static_cast<float>(1.0 / in->temperature - inv_t);
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

// Losses on the log-probabilities of sampled tokens: log-probability and its backward pass, the clipped policy objective with a KL
// term and its gradient in one pass, and the preference loss of pairs of sequences.
//
//   logp = (z_y - m) / t - log sum_j exp((z_j - m) / t),  m = max_j z_j,      dlogits_j = coef / t ([j = y] - q_j)
//   policy: coef = w (-A ratio [the unclipped term is the minimum] - kl_weight (exp(k) - 1))
//
// All of it is bound by memory, and the policy loss by a row's two passes too, the second of which comes from L2.  Measured: log-probabilities of
// 4096 x 32000 bfloat16 49 us (5.3 TB/s), their backward pass 84 us (6.2), the policy loss with its gradient 104 us (5.0 TB/s for one read and one
// write); 2049 x 50257 43, 69 and 96 us.
// Rows are taken relative to their largest logit before the division by t, as in distillation.  What a row's loss needs besides is a
// handful of scalars, which one thread computes in 64 bits: a log-probability of -10 in float would leave the ratio and the KL term
// (a difference of nearly equal numbers) only five digits.
#include <limits>

#include "logits_row.cuh"
#include "umma.cuh"

namespace collage {
namespace ops {

enum { kLogp = 0, kBackward = 1, kPolicy = 2 };

struct TokenArgs {
    const void* logits;
    const void* target;
    void* dlogits;
    const float* stats_in;
    const float* weight;                         // grad_logp, or the policy's row weights
    const float *old_logp, *ref_logp, *advantage;
    float *logp, *logp_rest, *stats, *loss, *kl;
    uint64_t ldz, ldd;
    double inv_t;
    float c, c_rest, inv_tf;                     // log2(e) / t rounded down and what it lacks, 1 / t
    float c_near;                                // log2(e) / t to nearest, for gradients: half a unit off, as the products with it are
    float clip_low, clip_high, kl_weight;        // bounds of the ratio
    uint32_t vocab, slice, cluster;              // slice: 16-byte vectors of a row for one block; cluster: blocks of a row
    int target_bytes;
};
constexpr uint32_t kTokenCluster = 8;

__device__ __forceinline__ int64_t index_at(const void* p, int bytes, uint64_t i) {
    return bytes == 8 ? static_cast<const int64_t*>(p)[i] : static_cast<const int32_t*>(p)[i];
}

// A row's scalars from its log-probability: the loss, its KL part, and the gradient of the log-probability.
struct PolicyRow {
    float loss, kl, coef;
};
__device__ __forceinline__ PolicyRow policy_row(const TokenArgs& a, uint64_t row, double logp, float w) {
    const float A = a.advantage[row];
    const float ratio = a.old_logp ? expf(static_cast<float>(logp - static_cast<double>(a.old_logp[row]))) : logp == logp ? 1.0f : NAN;
    const float free = ratio * A, held = fminf(fmaxf(ratio, a.clip_low), a.clip_high) * A;
    // (a NaN in either is the minimum)
    float loss = A == 0.0f ? 0.0f : held < free ? -held : -free, coef = A == 0.0f || held < free ? 0.0f : -free, kl = 0.0f;
    if (a.ref_logp) {
        const double k = static_cast<double>(a.ref_logp[row]) - logp;
        const float slope = static_cast<float>(expm1(k));
        kl = static_cast<float>(expm1(k) - k);
        if (a.kl_weight != 0.0f) {
            loss = __fmaf_rn(a.kl_weight, kl, loss);
            coef = __fmaf_rn(-a.kl_weight, slope, coef);
        }
    }
    return {w * loss, kl, w * coef};
}

// A warp's exponentials are relative to its largest logit so far, or to one that is less than 2^kLag times as likely, so that sums are hardly ever
// rescaled.  (A larger lag would need larger offsets, in which the smaller part of log2(e) / t is lost.)
constexpr float kLag = 1.0f;

// The hardware's 2^x is off by up to 1.5e-7, for x < 0 too low by 5.0e-8 on average (for x > 0 too high by 3.3e-8), and for a given x the same way
// each time: a row's sum would carry the average, or, of a row of few values, the errors of these.  So each thread takes its exponentials at an
// offset of its own, 2^(x + offset) with x + offset <= 0, and divides its sum by what the hardware gives for 2^offset.  The logit that all are
// relative to counts exactly 1; others have the difference of two errors, whose mean over offsets is 0 for any x, and a row's sum has the mean over
// its threads.  Multiples of the golden ratio, less their whole part, are evenly spread for 64 threads as for 256 and have no period
// in common with the hardware's intervals.
__device__ __forceinline__ float exp_offset(uint32_t thread) { return -kLag - static_cast<float>(thread * 0x9E3779B9u >> 8) * 0x1p-24f; }

// Sum of 2^offset exp((f - m) / t) over a vector, with log2(e) / t in two floats: what the first one lacks would shift the log-probabilities of
// all tokens the same way, which a sequence's sum adds up.  Sums go by twos, here and over vectors, so that a large term meets few roundings and
// equal terms meet none.
template <typename T>
__device__ __forceinline__ uint64_t offset_exps(const uint4& q, float m, float offset, const TokenArgs& a) {
    constexpr uint32_t kPairs = Vec<T>::kPairs;
    uint64_t f[kPairs];
    Vec<T>::unpack(q, f);
    const float minus_m = m == -INFINITY ? 0.0f : -m;
#pragma unroll
    for (uint32_t i = 0; i < kPairs; ++i) {
        const uint64_t d = add_pair(f[i], pair_of(minus_m));
        const float2 x = floats_of(fma_pair(d, pair_of(a.c), fma_pair(d, pair_of(a.c_rest), pair_of(offset))));
        f[i] = pair_of(fast_exp2(x.x), fast_exp2(x.y));
    }
    if constexpr (kPairs == 4)
        return add_pair(add_pair(f[0], f[1]), add_pair(f[2], f[3]));
    else
        return add_pair(f[0], f[1]);
}

// s / d for 2^-3 < d <= 1, by Newton's reciprocal and the quotient's remainder: 1 where they are equal.
__device__ __forceinline__ float quotient(float s, float d) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(d));
    const float q = s * r;
    return __fmaf_rn(__fmaf_rn(-q, d, s), r, q);
}

// What a sum relative to m is taken times to be relative to `to`: 2^x, x = (m - to) log2(e) / t = n + f with a whole n and |f| <= 1/2, and 2^f by its
// Taylor series, the sum of (f ln 2)^k / k!, whose terms from the eighth on are below 2^-27.  Correct but for a rounding or two, both ways.  (A sum
// of nothing is 0 or, of NaN alone, NaN; so it is times 0.)
__device__ __forceinline__ float factor_to(float m, float to, const TokenArgs& a) {
    if (m == to) return 1.0f;
    const float d = m - to, n = rintf(__fmaf_rn(d, a.c, d * a.c_rest));
    if (n < -125.0f) return 0.0f;
    const float f = __fmaf_rn(d, a.c_rest, __fmaf_rn(d, a.c, -n));
    float p = 1.52527338e-5f;                    // ln(2)^7 / 7!
    p = __fmaf_rn(p, f, 1.54035304e-4f);
    p = __fmaf_rn(p, f, 1.33335581e-3f);
    p = __fmaf_rn(p, f, 9.61812911e-3f);
    p = __fmaf_rn(p, f, 5.55041087e-2f);
    p = __fmaf_rn(p, f, 2.40226507e-1f);
    p = __fmaf_rn(p, f, 6.93147181e-1f);
    p = __fmaf_rn(p, f, 1.0f);
    return __uint_as_float(__float_as_uint(p) + (static_cast<uint32_t>(static_cast<int>(n)) << 23));
}

struct TokenShared {
    float2 warp[8];                      // what each warp's sum is relative to, and the sum
    float top[8];                        // its maximum
    float2 part[kTokenCluster];          // (maximum, sum) of each block of the cluster
    float coef, scale, at_target;
};

// A row by a cluster of blocks, each with a slice of it that it streams from global memory, once for maximum and sum and once for
// the gradient.  Log-probabilities with 2048 threads on an SM have 32 registers and spill a few; with 1536 they are as fast (2049 x 50257 42.4 us, not
// 42.5; 4096 x 32000 48.5, not 48.9; in float 81.0, not 87.5) but for rows of a turn or two (8192 x 8192 38.8, not 35.8).
template <typename T, int MODE, int THREADS>
__global__ void __launch_bounds__(THREADS, (MODE == kLogp ? 2048 : 1280) / THREADS) token_kernel(const __grid_constant__ TokenArgs a) {
    using V = Vec<T>;
    constexpr uint32_t kN = V::kN, kAhead = 4;
    __shared__ TokenShared sh;
    after_previous();
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = a.cluster > 1 ? (MODE == kBackward ? blockIdx.x % a.cluster : umma::cluster_rank()) : 0;
    const uint64_t row = blockIdx.x / a.cluster;
    const RowVectors<T> z(const_cast<T*>(static_cast<const T*>(a.logits)) + row * a.ldz, a.vocab);
    const RowVectors<T> dz(MODE != kLogp ? static_cast<T*>(a.dlogits) + row * a.ldd : nullptr, a.vocab);
    const uint32_t first = rank * a.slice, end = min(first + a.slice, z.count());        // this block's vectors
    const int64_t y = index_at(a.target, a.target_bytes, row);
    const float w = MODE == kLogp ? 1.0f : a.weight[row];
    const uint4 lowest = make_uint4(V::kLowest, V::kLowest, V::kLowest, V::kLowest);
    // Whole vectors of the slice; the row's first and last one may be cut.
    const uint32_t whole = first + (first < end && !z.inside(first)), whole_end = max(whole, end - (first < end && !z.inside(end - 1)));
    // Gradients of the slice; `value` turns a pair of logits into gradients.  Cut vectors, and rows whose gradients lie otherwise
    // in their vectors, go by elements.
    auto write_row = [&](bool read, auto&& value) {
        if (first >= end) return;
        auto by_elements = [&](uint32_t lo, uint32_t hi) {
#pragma unroll 1
            for (uint32_t e = lo + threadIdx.x; e < hi; e += THREADS) dz.row[e] = V::rounded(floats_of(value(pair_of(read ? V::value(z.row[e]) : 0.0f, 0.0f))).x);
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
        for (; v + (kAhead - 1) * THREADS < whole_end; v += THREADS * kAhead) {
            uint4 q[kAhead];
#pragma unroll
            for (uint32_t i = 0; i < kAhead; ++i) q[i] = read ? z.base[v + i * THREADS] : lowest;
#pragma unroll
            for (uint32_t i = 0; i < kAhead; ++i) put(v + i * THREADS, q[i]);
        }
#pragma unroll 1
        for (; v < whole_end; v += THREADS) put(v, read ? z.base[v] : lowest);
        if (whole > first) by_elements(lo, min(whole * kN - z.off, hi));
        if (whole_end < end) by_elements(whole_end * kN - z.off, hi);
    };
    if (y < 0 || y >= a.vocab || w == 0.0f) {           // not read
        if (MODE != kLogp) write_row(false, [](uint64_t) -> uint64_t { return 0; });
        if (MODE != kBackward && rank == 0 && threadIdx.x == 0) {
            if (a.logp) a.logp[row] = 0.0f;
            if (MODE == kLogp && a.logp_rest) a.logp_rest[row] = 0.0f;
            if (MODE == kLogp && a.stats) reinterpret_cast<float2*>(a.stats)[row] = make_float2(0.0f, 0.0f);
            if (MODE == kPolicy) a.loss[row] = 0.0f;
            if (MODE == kPolicy && a.kl) a.kl[row] = 0.0f;
        }
        return;
    }
    float m, scale, coef;
    float at_target = 0.0f;
    if (threadIdx.x == 0) at_target = V::value(z.row[y]);
    if (MODE == kBackward) {
        const float2 s = reinterpret_cast<const float2*>(a.stats_in)[row];
        m = s.x;
        scale = 1.0f / s.y;
        coef = w;
        __syncthreads();                                 // the target's logit has been read: it may be overwritten
    } else {
        if (a.cluster > 1) umma::cluster_arrive_all();                       // this block runs
        // maximum and sum of this thread's vectors, joined over the warp, the block and the cluster
        float from = -INFINITY;                 // what this warp's exponentials are relative to
        m = -INFINITY;
        uint64_t total = 0;
        const float offset = exp_offset(rank * THREADS + threadIdx.x);
        auto take = [&](const uint4 (&q)[kAhead]) {
            typename V::Most most = V::lowest();
#pragma unroll
            for (uint32_t i = 0; i < kAhead; ++i) most = V::most(most, q[i]);
            m = fmaxf(m, V::most_value(most));
            if (__any_sync(0xFFFFFFFFu, (m - from) * a.c > kLag)) {
                const float to = warp_max(m);
                total = mul_pair(total, pair_of(factor_to(from, to, a)));
                from = to;
            }
            uint64_t part[kAhead];
#pragma unroll
            for (uint32_t i = 0; i < kAhead; ++i) part[i] = offset_exps<T>(q[i], from, offset, a);
            total = add_pair(total, add_pair(add_pair(part[0], part[1]), add_pair(part[2], part[3])));
        };
        for (uint32_t v = whole + threadIdx.x; v - lane < whole_end; v += THREADS * kAhead) {          // (as many turns for all of a warp)
            uint4 q[kAhead];
#pragma unroll
            for (uint32_t i = 0; i < kAhead; ++i) q[i] = v + i * THREADS < whole_end ? z.base[v + i * THREADS] : lowest;
            take(q);
        }
        if (warp == 0 && (whole > first || whole_end < end)) {       // cut vectors: one thread for each
            uint4 q[kAhead] = {lowest, lowest, lowest, lowest};
            if (lane == 0 && whole > first) q[0] = z.edge(first);
            if (lane == 1 && whole_end < end) q[0] = z.edge(end - 1);
            take(q);
        }
        const float2 sums = floats_of(total);
        float sum = warp_sum(quotient(sums.x + sums.y, fast_exp2(offset)));
        m = warp_max(m);
        if (lane == 0) {
            sh.warp[warp] = make_float2(from, sum);
            sh.top[warp] = m;
        }
        __syncthreads();
        const float2 of_warp = lane < THREADS / 32 ? sh.warp[lane] : make_float2(-INFINITY, 0.0f);
        m = warp_max(lane < THREADS / 32 ? sh.top[lane] : -INFINITY);
        sum = warp_sum(of_warp.y * factor_to(of_warp.x, m, a));
        if (a.cluster > 1) {
            umma::cluster_wait_all();           // all blocks of the row run
            if (threadIdx.x < a.cluster) {
                const uint32_t to = umma::cluster_addr(&sh.part[rank], threadIdx.x);
                asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(to), "f"(m), "f"(sum) : "memory");
            }
            umma::cluster_sync_any();           // (also: the whole row has been read before any of it is overwritten)
            const float2 r = lane < a.cluster ? sh.part[lane] : make_float2(-INFINITY, 0.0f);
            m = warp_max(r.x);
            sum = warp_sum(r.y * factor_to(r.x, m, a));
        }
        if (m == -INFINITY) sum = NAN;          // a row without any number in it has no distribution
        scale = 1.0f / sum;
        coef = 0.0f;
        if (threadIdx.x == 0 && (MODE == kPolicy || rank == 0)) {
            const double logp = (static_cast<double>(at_target) - static_cast<double>(m)) * a.inv_t - log(static_cast<double>(sum));
            if (rank == 0 && a.logp) a.logp[row] = static_cast<float>(logp);
            if (MODE == kLogp && a.logp_rest) {      // (of an infinite one nothing is missing)
                const float rest = static_cast<float>(logp - static_cast<double>(static_cast<float>(logp)));
                a.logp_rest[row] = isinf(logp) ? 0.0f : rest;
            }
            if (MODE == kLogp && a.stats) reinterpret_cast<float2*>(a.stats)[row] = make_float2(m, sum);
            if (MODE == kPolicy) {
                const PolicyRow r = policy_row(a, row, logp, w);
                if (rank == 0) {
                    a.loss[row] = r.loss;
                    if (a.kl) a.kl[row] = r.kl;
                }
                sh.coef = r.coef;
            }
        }
        if (MODE == kLogp) return;
        __syncthreads();
        coef = sh.coef;
    }
    const float gain = coef * a.inv_tf;
    if (gain == 0.0f) {
        write_row(false, [](uint64_t) -> uint64_t { return 0; });
        return;
    }
    const float minus = -gain * scale;
    const uint64_t m2 = pair_of(-m, -m), c2 = pair_of(a.c_near, a.c_near), g2 = pair_of(minus, minus);
    write_row(true, [&](uint64_t f) {
        const float2 e = exps(f, m2, c2);
        return mul_pair(g2, pair_of(e.x, e.y));
    });
    const uint32_t vy = (static_cast<uint32_t>(y) + z.off) / kN;
    if (vy < first || vy >= end) return;
    __syncthreads();                        // the dense part is written; now the target over it
    if (threadIdx.x == 0) dz.row[y] = V::rounded(__fmaf_rn(minus, fast_exp2((at_target - m) * a.c_near), gain));
}

template <typename T, int MODE>
static collage_status_t launch_token_as(const TokenArgs& a, uint64_t rows, cudaStream_t s) {
    const uint32_t cluster = MODE == kBackward ? 1 : a.cluster;
    if (a.slice <= 256) return launch<&token_kernel<T, MODE, 64>>(rows * a.cluster, 64, cluster, 0, s, a);
    if (a.slice <= 1024) return launch<&token_kernel<T, MODE, 128>>(rows * a.cluster, 128, cluster, 0, s, a);
    return launch<&token_kernel<T, MODE, 256>>(rows * a.cluster, 256, cluster, 0, s, a);
}

template <int MODE>
static collage_status_t launch_token(TokenArgs& a, uint64_t rows, collage_dtype_t dtype, int sm_count, cudaStream_t s) {
    const uint32_t per_vector = dtype == COLLAGE_DTYPE_BF16 ? 8 : 4;
    const uint32_t vectors = (a.vocab + 2 * per_vector - 2) / per_vector;        // at the worst alignment
    a.cluster = 1;
    // few rows: more blocks for each, up to four on an SM in all and down to 512 vectors each
    while (a.cluster < kTokenCluster && rows * a.cluster * 2 <= 4ull * sm_count && vectors / a.cluster >= 1024) a.cluster *= 2;
    // Rows that are read twice: as many blocks for each as keep all rows under way in L2 (five blocks an SM).  1024 x 131072: 147 us without,
    // 120 with four each; 4096 x 32000 in float 234 and 202.  Of shorter rows more blocks cost more than they save (2049 x 50257: 95 and 100).
    if (MODE == kPolicy)
        while (a.cluster < kTokenCluster && 5ull * sm_count / a.cluster * vectors * 16 > (80ull << 20) && vectors / a.cluster >= 1024) a.cluster *= 2;
    a.slice = (vectors + a.cluster - 1) / a.cluster;
    return dtype == COLLAGE_DTYPE_BF16 ? launch_token_as<uint16_t, MODE>(a, rows, s) : launch_token_as<float, MODE>(a, rows, s);
}

// ------------------------------------------------------------------------------------------------------- preference ---

struct PreferenceArgs {
    const float *logp, *logp_rest, *ref_logp, *pair_weight;
    const void *target, *offsets;
    float *loss, *log_ratio, *grad_logp;
    uint64_t rows, pairs;
    int64_t vocab;
    double beta, margin, smoothing;
    int target_bytes, offset_bytes, average;
};
constexpr int kPreferenceThreads = 512;

// A pair by a block: sums over both sequences in 64 bits, then the loss and the gradient of each row.
__global__ void __launch_bounds__(kPreferenceThreads) preference_kernel(const __grid_constant__ PreferenceArgs a) {
    __shared__ double part[2][kPreferenceThreads / 32];
    __shared__ uint32_t number[2][kPreferenceThreads / 32];
    __shared__ float of_row[2];
    after_previous();
    const uint64_t p = blockIdx.x;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    auto edge = [&](uint64_t i) {
        const int64_t o = index_at(a.offsets, a.offset_bytes, i);
        return o < 0 ? 0ull : min(static_cast<uint64_t>(o), a.rows);
    };
    const uint64_t edges[3] = {edge(2 * p), edge(2 * p + 1), edge(2 * p + 2)};
    auto counts = [&](uint64_t i) {
        const int64_t y = index_at(a.target, a.target_bytes, i);
        return y >= 0 && y < a.vocab;
    };
    double sum[2] = {0.0, 0.0};
    uint32_t n[2] = {0, 0};
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        for (uint64_t i = edges[s] + threadIdx.x; i < edges[s + 1]; i += kPreferenceThreads) {
            if (!counts(i)) continue;
            sum[s] += static_cast<double>(a.logp[i]) + (a.logp_rest ? static_cast<double>(a.logp_rest[i]) : 0.0) - (a.ref_logp ? static_cast<double>(a.ref_logp[i]) : 0.0);
            ++n[s];
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum[s] += __shfl_xor_sync(0xFFFFFFFFu, sum[s], o);
        n[s] = __reduce_add_sync(0xFFFFFFFFu, n[s]);
        if (lane == 0) {
            part[s][warp] = sum[s];
            number[s][warp] = n[s];
        }
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        double per[2];
        for (int s = 0; s < 2; ++s) {
            sum[s] = 0.0;
            n[s] = 0;
            for (int k = 0; k < kPreferenceThreads / 32; ++k) {
                sum[s] += part[s][k];
                n[s] += number[s][k];
            }
            per[s] = a.average && n[s] > 1 ? 1.0 / n[s] : 1.0;
        }
        const double log_ratio = sum[0] * per[0] - sum[1] * per[1], h = a.beta * log_ratio - a.margin;
        const double w = a.pair_weight ? a.pair_weight[p] : 1.0;
        // -log sigmoid(h) = log1p(exp(-|h|)) + max(-h, 0); terms of factor 0 are left out (they may be infinite)
        const double both = log1p(exp(-fabs(h))), small = exp(-fabs(h)) / (1.0 + exp(-fabs(h)));       // sigmoid(-|h|)
        double loss = 0.0, slope = 0.0;                                                                  // d loss / d h
        if (a.smoothing != 1.0) {
            loss += (1.0 - a.smoothing) * (both + (h < 0.0 ? -h : h == h ? 0.0 : h));
            slope -= (1.0 - a.smoothing) * (h < 0.0 ? 1.0 - small : small);
        }
        if (a.smoothing != 0.0) {
            loss += a.smoothing * (both + (h > 0.0 ? h : h == h ? 0.0 : h));
            slope += a.smoothing * (h > 0.0 ? 1.0 - small : small);
        }
        // a pair of weight 0 takes no part, whatever its log-probabilities are
        a.loss[p] = w == 0.0 ? 0.0f : static_cast<float>(w * loss);
        if (a.log_ratio) a.log_ratio[p] = static_cast<float>(log_ratio);
        of_row[0] = w == 0.0 ? 0.0f : static_cast<float>(w * a.beta * slope * per[0]);
        of_row[1] = w == 0.0 ? 0.0f : static_cast<float>(-w * a.beta * slope * per[1]);
    }
    if (!a.grad_logp) return;
    __syncthreads();
#pragma unroll
    for (int s = 0; s < 2; ++s)
        for (uint64_t i = edges[s] + threadIdx.x; i < edges[s + 1]; i += kPreferenceThreads) a.grad_logp[i] = counts(i) ? of_row[s] : 0.0f;
    // rows of no sequence
    if (p == 0)
        for (uint64_t i = threadIdx.x; i < edges[0]; i += kPreferenceThreads) a.grad_logp[i] = 0.0f;
    if (p + 1 == a.pairs)
        for (uint64_t i = edges[2] + threadIdx.x; i < a.rows; i += kPreferenceThreads) a.grad_logp[i] = 0.0f;
}

// Everything the entry points over logits check alike; `read` and `written` are their float arrays, of `per` values a row.
struct RowArray {
    const float* p;
    uint64_t per;
};
static collage_status_t prepare_tokens(const collage_tokens_t* in, const RowArray (&read)[4], const RowArray (&written)[3], const collage_matrix_t* dlogits,
                                       TokenArgs* out, DeviceInfo* dev) {
    const uint32_t size = in->logits_dtype == COLLAGE_DTYPE_BF16 ? 2 : 4;
    if (in->logits_dtype != COLLAGE_DTYPE_BF16 && in->logits_dtype != COLLAGE_DTYPE_F32) return COLLAGE_ERR_ARG;
    if (in->target_bytes != 4 && in->target_bytes != 8) return COLLAGE_ERR_ARG;
    if (!(std::isfinite(in->temperature) && in->temperature > 0.0)) return COLLAGE_ERR_ARG;
    const double inv_t = 1.0 / in->temperature;
    // log2(e) / t rounded down, so that what it lacks is above 0: a logit of -infinity, times either, is -infinity
    const double exact_c = inv_t * 1.4426950408889634074;
    const float t = static_cast<float>(in->temperature), near_c = static_cast<float>(exact_c), c = near_c < exact_c ? near_c : std::nextafterf(near_c, 0.0f);
    if (!(t > 0.0f && std::isfinite(t) && static_cast<float>(inv_t) > 0.0f && std::isfinite(near_c) && c > 0.0f)) return COLLAGE_ERR_ARG;
    if (dlogits && !same_shape(dlogits, &in->logits)) return COLLAGE_ERR_ARG;
    collage_status_t st = check_matrix(&in->logits, size);
    if (st == COLLAGE_OK && dlogits) st = check_matrix(dlogits, size);
    if (st != COLLAGE_OK) return st;
    const uint64_t rows = in->logits.rows;
    if (!in->target && rows) return COLLAGE_ERR_NULL;
    if (reinterpret_cast<uintptr_t>(in->target) % in->target_bytes) return COLLAGE_ERR_ARG;
    AliasCheck alias;
    const int iz = alias.add(span_of(&in->logits, size), false);
    alias.add(span_of(in->target, in->target_bytes * rows), false);
    for (const RowArray& r : read) {
        if (reinterpret_cast<uintptr_t>(r.p) % (4 * r.per)) return COLLAGE_ERR_ARG;
        if (r.p) alias.add(span_of(r.p, 4 * r.per * rows), false);
    }
    for (const RowArray& r : written) {
        if (reinterpret_cast<uintptr_t>(r.p) % (4 * r.per)) return COLLAGE_ERR_ARG;
        if (r.p) alias.add(span_of(r.p, 4 * r.per * rows), true);
    }
    const int id = dlogits ? alias.add(span_of(dlogits, size), true) : -1;
    const int pairs[1][2] = {{id, iz}};
    if (alias.clash(pairs)) return COLLAGE_ERR_ALIAS;
    if ((st = current_device(dev)) != COLLAGE_OK) return st;
    *out = {};
    out->logits = in->logits.data;
    out->ldz = in->logits.ld;
    out->target = in->target;
    out->target_bytes = static_cast<int>(in->target_bytes);
    if (dlogits) { out->dlogits = dlogits->data; out->ldd = dlogits->ld; }
    out->vocab = static_cast<uint32_t>(in->logits.cols);
    out->inv_t = inv_t;
    out->inv_tf = static_cast<float>(inv_t);
    out->c = c;
    out->c_near = near_c;
    out->c_rest = std::max(static_cast<float>(exact_c - c), std::numeric_limits<float>::denorm_min());
    return COLLAGE_OK;
}

}  // namespace ops
}  // namespace collage

using namespace collage;
using namespace collage::ops;

extern "C" {

collage_status_t collage_token_logp(const collage_tokens_t* in, float* logp, float* logp_rest, float* stats, void* stream) {
    if (!in || (!logp && in->logits.rows)) return COLLAGE_ERR_NULL;
    TokenArgs a;
    DeviceInfo dev;
    const collage_status_t st = prepare_tokens(in, {{nullptr, 1}, {nullptr, 1}, {nullptr, 1}, {nullptr, 1}}, {{logp, 1}, {stats, 2}, {logp_rest, 1}}, nullptr, &a, &dev);
    if (st != COLLAGE_OK || in->logits.rows == 0) return st;
    a.logp = logp;
    a.logp_rest = logp_rest;
    a.stats = stats;
    return launch_token<kLogp>(a, in->logits.rows, in->logits_dtype, dev.sm_count, static_cast<cudaStream_t>(stream));
}

collage_status_t collage_token_logp_backward(const collage_tokens_t* in, const float* stats, const float* grad_logp,
                                             const collage_matrix_t* dlogits, void* stream) {
    if (!in || !dlogits || ((!stats || !grad_logp) && in->logits.rows)) return COLLAGE_ERR_NULL;
    TokenArgs a;
    DeviceInfo dev;
    const collage_status_t st = prepare_tokens(in, {{stats, 2}, {grad_logp, 1}, {nullptr, 1}, {nullptr, 1}}, {{nullptr, 1}, {nullptr, 1}, {nullptr, 1}}, dlogits, &a, &dev);
    if (st != COLLAGE_OK || in->logits.rows == 0 || in->logits.cols == 0) return st;
    a.stats_in = stats;
    a.weight = grad_logp;
    return launch_token<kBackward>(a, in->logits.rows, in->logits_dtype, dev.sm_count, static_cast<cudaStream_t>(stream));
}

collage_status_t collage_policy_loss_and_grad(const collage_tokens_t* in, const collage_policy_t* policy, float* loss, float* logp, float* kl,
                                              const collage_matrix_t* dlogits, void* stream) {
    if (!in || !policy || !dlogits || ((!loss || !policy->advantage || !policy->row_weight) && in->logits.rows)) return COLLAGE_ERR_NULL;
    const float low = static_cast<float>(1.0 - policy->clip_low), high = static_cast<float>(1.0 + policy->clip_high), kl_weight = static_cast<float>(policy->kl_weight);
    if (!(policy->clip_low >= 0.0 && policy->clip_low <= 1.0 && policy->clip_high >= 0.0 && policy->kl_weight >= 0.0 && std::isfinite(kl_weight))) return COLLAGE_ERR_ARG;
    if (!policy->ref_logp && (kl || kl_weight != 0.0f)) return COLLAGE_ERR_ARG;
    TokenArgs a;
    DeviceInfo dev;
    const collage_status_t st = prepare_tokens(in, {{policy->old_logp, 1}, {policy->ref_logp, 1}, {policy->advantage, 1}, {policy->row_weight, 1}},
                                               {{loss, 1}, {logp, 1}, {kl, 1}}, dlogits, &a, &dev);
    if (st != COLLAGE_OK || in->logits.rows == 0) return st;
    a.weight = policy->row_weight;
    a.old_logp = policy->old_logp;
    a.ref_logp = policy->ref_logp;
    a.advantage = policy->advantage;
    a.clip_low = low;
    a.clip_high = high;
    a.kl_weight = kl_weight;
    a.loss = loss;
    a.logp = logp;
    a.kl = kl;
    return launch_token<kPolicy>(a, in->logits.rows, in->logits_dtype, dev.sm_count, static_cast<cudaStream_t>(stream));
}

collage_status_t collage_preference_loss(const collage_preference_t* in, float* loss, float* log_ratio, float* grad_logp, void* stream) {
    if (!in) return COLLAGE_ERR_NULL;
    if (in->rows > kMaxExtent || in->pairs > kMaxExtent / 2 || in->vocab > kMaxExtent) return COLLAGE_ERR_LIMIT;
    auto fits = [](double v) { return std::isfinite(v) && std::isfinite(static_cast<float>(v)); };
    if (!fits(in->beta) || !fits(in->margin) || !(in->label_smoothing >= 0.0 && in->label_smoothing <= 1.0)) return COLLAGE_ERR_ARG;
    if ((in->target_bytes != 4 && in->target_bytes != 8) || (in->offset_bytes != 4 && in->offset_bytes != 8)) return COLLAGE_ERR_ARG;
    if ((in->rows && (!in->logp || !in->target)) || (in->pairs && (!loss || !in->offsets))) return COLLAGE_ERR_NULL;
    auto off = [](const void* p, uint64_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes != 0; };
    if (off(in->logp, 4) || off(in->logp_rest, 4) || off(in->ref_logp, 4) || off(in->pair_weight, 4) || off(loss, 4) || off(log_ratio, 4) || off(grad_logp, 4) ||
        off(in->target, in->target_bytes) || off(in->offsets, in->offset_bytes))
        return COLLAGE_ERR_ARG;
    AliasCheck alias;
    alias.add(span_of(in->logp, 4 * in->rows), false);
    alias.add(span_of(in->logp_rest, 4 * in->rows), false);
    alias.add(span_of(in->ref_logp, 4 * in->rows), false);
    alias.add(span_of(in->target, in->target_bytes * in->rows), false);
    alias.add(span_of(in->offsets, in->offset_bytes * (2 * in->pairs + 1)), false);
    alias.add(span_of(in->pair_weight, 4 * in->pairs), false);
    alias.add(span_of(loss, 4 * in->pairs), true);
    alias.add(span_of(log_ratio, 4 * in->pairs), true);
    alias.add(span_of(grad_logp, 4 * in->rows), true);
    if (alias.clash()) return COLLAGE_ERR_ALIAS;
    DeviceInfo dev;
    if (const collage_status_t st = current_device(&dev); st != COLLAGE_OK) return st;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (in->pairs == 0)
        return !grad_logp || !in->rows || cudaMemsetAsync(grad_logp, 0, 4 * in->rows, s) == cudaSuccess ? COLLAGE_OK : COLLAGE_ERR_CUDA;
    PreferenceArgs a = {};
    a.logp = in->logp;
    a.logp_rest = in->logp_rest;
    a.ref_logp = in->ref_logp;
    a.pair_weight = in->pair_weight;
    a.target = in->target;
    a.offsets = in->offsets;
    a.loss = loss;
    a.log_ratio = log_ratio;
    a.grad_logp = grad_logp;
    a.rows = in->rows;
    a.pairs = in->pairs;
    a.vocab = static_cast<int64_t>(in->vocab);
    a.beta = in->beta;
    a.margin = in->margin;
    a.smoothing = in->label_smoothing;
    a.target_bytes = static_cast<int>(in->target_bytes);
    a.offset_bytes = static_cast<int>(in->offset_bytes);
    a.average = in->average != 0;
    return launch<&preference_kernel>(in->pairs, kPreferenceThreads, 1, 0, s, a);
}

}  // extern "C"

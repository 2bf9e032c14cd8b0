// Gated feed-forward projections: h = a(x w_gate^T) * (x w_up^T), the backward pass, and the same with e4m3 operands.
#include "product_any.cuh"

namespace collage {

cudaError_t read_clear_product_fault(unsigned int* out) {
    const unsigned int zero = 0;
    const cudaError_t e = cudaMemcpyFromSymbol(out, ops::g_product_fault, sizeof *out);
    return e != cudaSuccess || *out == 0 ? e : cudaMemcpyToSymbol(ops::g_product_fault, &zero, sizeof zero);
}

namespace ops {

struct GateArgs {
    const uint16_t *dh, *gate, *up;
    uint16_t *dgate, *dup;
    uint64_t lddh, ldg, ldu, lddg, lddu, cols;
    int activation;
};

__global__ void __launch_bounds__(256) gate_backward_any_kernel(const __grid_constant__ GateArgs a) {
    after_previous();
    const uint64_t row = blockIdx.x;
    for (uint64_t j = threadIdx.x; j < a.cols; j += 256) {
        const float dh = bf16_value(a.dh[row * a.lddh + j]), u = bf16_value(a.up[row * a.ldu + j]);
        const float2 as = activate_and_slope(a.activation, bf16_value(a.gate[row * a.ldg + j]));
        a.dgate[row * a.lddg + j] = to_bf16(dh * u * as.y);
        a.dup[row * a.lddu + j] = to_bf16(dh * as.x);
    }
}

// The same on rows of whole 16-byte vectors: a vector a thread and turn, the next one's loads sent before this one's results.
__global__ void __launch_bounds__(256) gate_backward_kernel(const __grid_constant__ GateArgs a, uint64_t rows) {
    after_previous();
    const uint64_t vectors = a.cols >> 3, total = rows * vectors, step = gridDim.x * 256ull;
    auto at = [](const uint16_t* p, uint64_t ld, uint64_t row, uint64_t v) { return reinterpret_cast<const uint4*>(p + row * ld) + v; };
    uint4 next[3];
    uint64_t row = 0, v = 0;
    auto load = [&](uint64_t i) {
        row = i / vectors;
        v = i - row * vectors;
        next[0] = __ldcs(at(a.dh, a.lddh, row, v));
        next[1] = *at(a.gate, a.ldg, row, v);
        next[2] = *at(a.up, a.ldu, row, v);
    };
    uint64_t i = blockIdx.x * 256ull + threadIdx.x;
    if (i < total) load(i);
    for (; i < total; i += step) {
        const uint32_t d[4] = {next[0].x, next[0].y, next[0].z, next[0].w}, g[4] = {next[1].x, next[1].y, next[1].z, next[1].w},
                       u[4] = {next[2].x, next[2].y, next[2].z, next[2].w};
        const uint64_t this_row = row, this_v = v;
        if (i + step < total) load(i + step);
        uint32_t dg[4], du[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float2 lo = activate_and_slope(a.activation, bf16_lo(g[e])), hi = activate_and_slope(a.activation, bf16_hi(g[e]));
            dg[e] = pack_bf16(bf16_lo(d[e]) * bf16_lo(u[e]) * lo.y, bf16_hi(d[e]) * bf16_hi(u[e]) * hi.y);
            du[e] = pack_bf16(bf16_lo(d[e]) * lo.x, bf16_hi(d[e]) * hi.x);
        }
        reinterpret_cast<uint4*>(a.dgate + this_row * a.lddg)[this_v] = make_uint4(dg[0], dg[1], dg[2], dg[3]);
        reinterpret_cast<uint4*>(a.dup + this_row * a.lddu)[this_v] = make_uint4(du[0], du[1], du[2], du[3]);
    }
}

// ---- tensor-map path -------------------------------------------------------------------------------------------------

using EncodeTiled = decltype(&cuTensorMapEncodeTiled);

static EncodeTiled encode_tiled() {
    static std::atomic<void*> cached{nullptr};
    void* fn = cached.load(std::memory_order_acquire);
    if (!fn) {
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &found) != cudaSuccess ||
            found != cudaDriverEntryPointSuccess)
            return nullptr;
        cached.store(fn, std::memory_order_release);
    }
    return reinterpret_cast<EncodeTiled>(fn);
}

// The matrix as a two-dimensional tensor read in boxes of box_cols x box_rows; outside it a load gives zeros and a store
// writes nothing.
static bool make_map(CUtensorMap* map, const collage_matrix_t* m, bool bytes, uint32_t box_cols, uint32_t box_rows, bool output) {
    const EncodeTiled encode = encode_tiled();
    if (!encode) return false;
    const cuuint64_t size = bytes ? 1 : 2;
    const cuuint64_t dims[2] = {m->cols, m->rows};
    const cuuint64_t strides[1] = {m->rows > 1 ? m->ld * size : (m->cols * size + 15) / 16 * 16};
    const cuuint32_t box[2] = {box_cols, box_rows}, one[2] = {1, 1};
    return encode(map, bytes ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, m->data, dims, strides, box, one,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, output ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B,
                  CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Can tensor maps describe it?  Rows on 16 bytes and of whole 16 bytes (a tile store writes no less), a stride below 2^40 bytes.
static bool mappable(const collage_matrix_t* m, uint32_t elem_bytes) {
    return rows_aligned(m, elem_bytes, 16) && m->cols * elem_bytes % 16 == 0 && (m->rows <= 1 || m->ld * elem_bytes < (1ull << 40));
}

template <bool E4M3, bool A_MN, bool GATED>
static collage_status_t launch_tiles(TileArgs& t, int sm_count, cudaStream_t s) {
    constexpr uint32_t out_cols = GATED ? 128 : 256;
    t.m_tiles = (t.m + 255) / 256;
    t.n_tiles = (t.n + out_cols - 1) / out_cols;
    const uint64_t tiles = static_cast<uint64_t>(t.problems) * t.m_tiles * t.n_tiles;
    if (tiles >= (1ull << 31)) return COLLAGE_ERR_LIMIT;
    t.group = 8;                        // (4, 8 and 16 rows of tiles at a time make no difference)
    return launch<&tile_kernel<E4M3, A_MN, GATED>>(std::min<uint64_t>(tiles, sm_count / 2) * 2, kTileThreads, 2, kTileSmem, s, t);
}

template <bool E4M3, bool A_MN, bool GATED, int NT>
static collage_status_t launch_slim_as(SlimArgs& t, uint64_t blocks, int sm_count, cudaStream_t s) {
    // (larger clusters of blocks that need an SM each leave SMs of a cluster's part of the GPU unused, and then take a second turn)
    const bool alone = blocks <= static_cast<uint64_t>(sm_count) && t.split <= 2;
    t.stages = std::min(kMaxSlimStages, slim_stages<NT>(alone));
    return launch<&slim_kernel<E4M3, A_MN, GATED, NT>>(blocks, kSlimThreads, t.split, slim_smem<NT>(alone), s, t);
}

// The most parts that a sum over `blocks` blocks of K is split into: at least eight blocks each.
static uint32_t most_split(uint32_t blocks) { return blocks >= 64 ? 8 : blocks >= 32 ? 4 : blocks >= 16 ? 2 : 1; }

// Tokens of a slim tile: all of them up to 128, fewer where even with K split a third of the SMs would be left without a tile
// (there are `weight_tiles` for each tile of tokens).  333 x 768 x 2048 forward: 10.9 us with 64 tokens, 14.4 with 128; but its dx, whose K
// can be split, loses by narrow tiles, which read the weights more often (160 x 4096 x 11008: 120 us against 55).
static uint32_t slim_tokens(uint64_t tokens, uint64_t weight_tiles, uint32_t blocks, int sm_count) {
    uint32_t nt = tokens <= 16 ? 16 : tokens <= 32 ? 32 : tokens <= 64 ? 64 : 128;
    while (nt > 32 && tokens > nt / 2 && (tokens + nt - 1) / nt * weight_tiles * most_split(blocks) * 3 < 2ull * sm_count) nt /= 2;
    return nt;
}

// The sum over K is split until there is a block for every SM, as long as each has eight blocks of K; of the narrowest tiles,
// three of which fit an SM, once more where enough of K is left (one token x 4096 x 11008: 33 against 35 us).
template <bool E4M3, bool A_MN, bool GATED>
static collage_status_t launch_slim(SlimArgs& t, uint32_t nt, uint64_t weight_tiles, int sm_count, cudaStream_t s) {
    const uint32_t blocks = t.terms * t.k_blocks;
    t.token_tiles = (t.n + nt - 1) / nt;
    const uint64_t tiles = t.token_tiles * weight_tiles;
    t.split = 1;
    while (t.split < most_split(blocks) && tiles * t.split < static_cast<uint64_t>(sm_count)) t.split *= 2;
    if (nt == 16 && t.split < 8 && tiles * t.split < 2ull * sm_count && blocks / (2 * t.split) >= 24) t.split *= 2;
    switch (nt) {
        case 16: return launch_slim_as<E4M3, A_MN, GATED, 16>(t, tiles * t.split, sm_count, s);
        case 32: return launch_slim_as<E4M3, A_MN, GATED, 32>(t, tiles * t.split, sm_count, s);
        case 64: return launch_slim_as<E4M3, A_MN, GATED, 64>(t, tiles * t.split, sm_count, s);
        default: return launch_slim_as<E4M3, A_MN, GATED, 128>(t, tiles * t.split, sm_count, s);
    }
}

// Slim tiles where there are few tokens, or too few pairs' tiles to keep the GPU busy (at 700 x 4096 x 11008 dx has 48 of them
// for 74 pairs: 115 us against 160 in slim tiles; at 384 it has 32: 90 us in slim tiles against 100).
static bool slim(uint64_t tokens, uint64_t pair_tiles, int sm_count) {
    return tokens <= 128 || pair_tiles * 18 < 5ull * sm_count;
}

// The forward products with 16-byte aligned rows.
template <bool E4M3>
static collage_status_t tiles_forward(const collage_matrix_t* x, const collage_matrix_t* wg, const collage_matrix_t* wu,
                                      const collage_matrix_t* h, const collage_matrix_t* gate, const collage_matrix_t* up,
                                      const float* const (&scales)[3], int activation, int sm_count, cudaStream_t s) {
    const uint32_t k = E4M3 ? 128 : 64;
    const uint32_t k_blocks = static_cast<uint32_t>((x->cols + k - 1) / k);
    const collage_matrix_t* outs[3] = {h, gate, up};
    if (slim(x->rows, (x->rows + 255) / 256 * ((h->cols + 127) / 128), sm_count)) {
        SlimArgs t = {};
        const uint64_t weight_tiles = (h->cols + 63) / 64;
        const uint32_t nt = slim_tokens(x->rows, weight_tiles, k_blocks, sm_count);
        if (!(make_map(&t.a[0], wg, E4M3, k, 64, false) && make_map(&t.a[1], wu, E4M3, k, 64, false) &&
              make_map(&t.b[0], x, E4M3, k, nt, false)))
            return COLLAGE_ERR_CUDA;
        for (int i = 0; i < 3 && outs[i]; ++i) {
            t.out[i] = static_cast<uint16_t*>(outs[i]->data);
            t.ldo[i] = outs[i]->ld;
        }
        t.token_scale = scales[0];
        t.row_scale[0] = scales[1];
        t.row_scale[1] = scales[2];
        t.m = static_cast<uint32_t>(h->cols);
        t.n = static_cast<uint32_t>(x->rows);
        t.k_blocks = k_blocks;
        t.terms = 1;
        t.keep = gate != nullptr;
        t.activation = activation;
        return launch_slim<E4M3, false, true>(t, nt, weight_tiles, sm_count, s);
    }
    TileArgs t = {};
    bool ok = make_map(&t.a[0], x, E4M3, k, 128, false) && make_map(&t.b[0], wg, E4M3, k, 128, false) && make_map(&t.b[1], wu, E4M3, k, 128, false);
    for (int i = 0; i < 3 && outs[i]; ++i) ok = ok && make_map(&t.out[i], outs[i], false, kUnitCols, 32, true);
    if (!ok) return COLLAGE_ERR_CUDA;
    t.a[1] = t.a[0];
    t.a_scale = scales[0];
    t.b_scale[0] = scales[1];
    t.b_scale[1] = scales[2];
    t.m = static_cast<uint32_t>(x->rows);
    t.n = static_cast<uint32_t>(wg->rows);
    t.problems = t.terms = 1;
    t.k_blocks = k_blocks;
    t.keep = gate != nullptr;
    t.activation = activation;
    return launch_tiles<E4M3, false, true>(t, sm_count, s);
}

static bool slim_dx(const collage_matrix_t* dx, int sm_count) {
    return slim(dx->rows, (dx->rows + 255) / 256 * ((dx->cols + 255) / 256), sm_count);
}
// The arguments of dx = dgate w_gate + dup w_up in slim tiles of `nt` tokens.
static bool slim_dx_args(SlimArgs& t, uint32_t& nt, const collage_matrix_t* dgate, const collage_matrix_t* dup, const collage_matrix_t* wg,
                         const collage_matrix_t* wu, const collage_matrix_t* dx, int sm_count) {
    t.k_blocks = static_cast<uint32_t>((dgate->cols + 63) / 64);
    t.terms = 2;
    nt = slim_tokens(dx->rows, (dx->cols + 127) / 128, 2 * t.k_blocks, sm_count);
    t.out[0] = static_cast<uint16_t*>(dx->data);
    t.ldo[0] = dx->ld;
    t.m = static_cast<uint32_t>(dx->cols);
    t.n = static_cast<uint32_t>(dx->rows);
    return make_map(&t.a[0], wg, false, 64, 64, false) && make_map(&t.a[1], wu, false, 64, 64, false) &&
           make_map(&t.b[0], dgate, false, 64, nt, false) && make_map(&t.b[1], dup, false, 64, nt, false);
}

// Both gradients in one launch pay where each is bound by its latencies: 333 x 768 x 2048 backward 21.0 us against 28.4, 2 x 1512 x
// 2136 19.6 against 22.4; but 1000 x 1024 x 2816 49 against 43, whose weight gradients the pairs' tiles make faster.
static bool small_layer(uint64_t tokens, const collage_matrix_t* dw, int sm_count) {
    return tokens <= 512 && 2 * ((dw->rows + 127) / 128) * ((dw->cols + 127) / 128) <= 3ull * sm_count;
}
// dx, dw_gate and dw_up of a small layer in one launch.
template <int NT>
static collage_status_t launch_slim_backward(SlimArgs& dx, SlimArgs& dw, uint64_t dx_tiles, int sm_count, cudaStream_t s) {
    const uint32_t blocks = dx.terms * dx.k_blocks;
    dx.split = 1;
    while (dx.split < most_split(blocks) && dx_tiles * dx.split < static_cast<uint64_t>(sm_count)) dx.split *= 2;
    dx.stages = std::min(kMaxSlimStages, slim_stages<NT>(false));
    dw.split = 1;
    dw.stages = slim_stages<128>(false);
    const uint64_t dw_tiles = 2ull * dw.token_tiles * ((dw.m + 127) / 128), dx_blocks = dx_tiles * dx.split;
    const uint64_t all = dx_blocks + (dw_tiles + dx.split - 1) / dx.split * dx.split;
    return launch<&slim_backward_kernel<NT>>(all, kSlimThreads, dx.split, std::max(slim_smem<NT>(false), slim_smem<128>(false)), s, dx, dw,
                                             static_cast<uint32_t>(dx_blocks), static_cast<uint32_t>(dw_tiles));
}
static collage_status_t slim_backward(const collage_matrix_t* dgate, const collage_matrix_t* dup, const collage_matrix_t* x,
                                      const collage_matrix_t* wg, const collage_matrix_t* wu, const collage_matrix_t* dx,
                                      const collage_matrix_t* dwg, const collage_matrix_t* dwu, int sm_count, cudaStream_t s) {
    SlimArgs a = {}, b = {};
    uint32_t nt;
    if (!(slim_dx_args(a, nt, dgate, dup, wg, wu, dx, sm_count) && make_map(&b.a[0], x, false, 64, 64, false) &&
          make_map(&b.b[0], dgate, false, 64, 64, false) && make_map(&b.b[1], dup, false, 64, 64, false)))
        return COLLAGE_ERR_CUDA;
    const collage_matrix_t* outs[2] = {dwg, dwu};
    for (int i = 0; i < 2; ++i) {
        b.out[i] = static_cast<uint16_t*>(outs[i]->data);
        b.ldo[i] = outs[i]->ld;
    }
    b.m = static_cast<uint32_t>(dwg->cols);
    b.n = static_cast<uint32_t>(dwg->rows);
    b.k_blocks = static_cast<uint32_t>((x->rows + 63) / 64);
    b.terms = 1;
    b.token_tiles = (b.n + 127) / 128;
    a.token_tiles = (a.n + nt - 1) / nt;
    const uint64_t dx_tiles = static_cast<uint64_t>(a.token_tiles) * ((a.m + 127) / 128);
    switch (nt) {
        case 16: return launch_slim_backward<16>(a, b, dx_tiles, sm_count, s);
        case 32: return launch_slim_backward<32>(a, b, dx_tiles, sm_count, s);
        case 64: return launch_slim_backward<64>(a, b, dx_tiles, sm_count, s);
        default: return launch_slim_backward<128>(a, b, dx_tiles, sm_count, s);
    }
}

// dx = dgate w_gate + dup w_up
static collage_status_t tiles_dx(const collage_matrix_t* dgate, const collage_matrix_t* dup, const collage_matrix_t* wg,
                                 const collage_matrix_t* wu, const collage_matrix_t* dx, int sm_count, cudaStream_t s) {
    if (slim_dx(dx, sm_count)) {
        SlimArgs t = {};
        uint32_t nt;
        if (!slim_dx_args(t, nt, dgate, dup, wg, wu, dx, sm_count)) return COLLAGE_ERR_CUDA;
        return launch_slim<false, true, false>(t, nt, (dx->cols + 127) / 128, sm_count, s);
    }
    const uint32_t k_blocks = static_cast<uint32_t>((dgate->cols + 63) / 64);
    TileArgs t = {};
    if (!(make_map(&t.a[0], dgate, false, 64, 128, false) && make_map(&t.a[1], dup, false, 64, 128, false) &&
          make_map(&t.b[0], wg, false, 64, 64, false) && make_map(&t.b[1], wu, false, 64, 64, false) &&
          make_map(&t.out[0], dx, false, kUnitCols, 32, true)))
        return COLLAGE_ERR_CUDA;
    t.m = static_cast<uint32_t>(dx->rows);
    t.n = static_cast<uint32_t>(dx->cols);
    t.problems = 1;
    t.terms = 2;
    t.k_blocks = k_blocks;
    return launch_tiles<false, false, false>(t, sm_count, s);
}

// dw_gate = dgate^T x and dw_up = dup^T x
static collage_status_t tiles_dw(const collage_matrix_t* dgate, const collage_matrix_t* dup, const collage_matrix_t* x,
                                 const collage_matrix_t* dwg, const collage_matrix_t* dwu, int sm_count, cudaStream_t s) {
    TileArgs t = {};
    if (!(make_map(&t.a[0], dgate, false, 64, 64, false) && make_map(&t.a[1], dup, false, 64, 64, false) &&
          make_map(&t.b[0], x, false, 64, 64, false) && make_map(&t.out[0], dwg, false, kUnitCols, 32, true) &&
          make_map(&t.out[1], dwu, false, kUnitCols, 32, true)))
        return COLLAGE_ERR_CUDA;
    t.b[1] = t.b[0];
    t.m = static_cast<uint32_t>(dwg->rows);
    t.n = static_cast<uint32_t>(dwg->cols);
    t.problems = 2;
    t.terms = 1;
    t.k_blocks = static_cast<uint32_t>((x->rows + 63) / 64);
    return launch_tiles<false, true, false>(t, sm_count, s);
}

// ---- any alignment ---------------------------------------------------------------------------------------------------

static Operand by_row(const collage_matrix_t* m) { return {m->data, m->ld, 1}; }        // i = row of the matrix
static Operand by_col(const collage_matrix_t* m) { return {m->data, 1, m->ld}; }        // i = column

// p's operands, outputs, scales, m, n, k and terms are set.
template <bool E4M3, bool GATED>
static collage_status_t launch_any(AnyArgs& p, int sm_count, cudaStream_t s) {
    if (p.m == 0 || p.n == 0) return COLLAGE_OK;
    const uint32_t nt = p.n <= 32 ? 32 : 128, k = E4M3 ? 128 : 64;
    p.token_tiles = (p.n + nt - 1) / nt;
    p.k_blocks = (p.k + k - 1) / k;
    const uint64_t tiles = static_cast<uint64_t>(p.token_tiles) * ((p.m + (GATED ? 63ull : 127ull)) / (GATED ? 64 : 128));
    p.split = 1;
    while (p.split < most_split(p.terms * p.k_blocks) && tiles * p.split < static_cast<uint64_t>(sm_count)) p.split *= 2;
    return nt == 32 ? launch<&any_kernel<E4M3, GATED, 32>>(tiles * p.split, kAnyThreads, p.split, any_smem<32>(), s, p)
                    : launch<&any_kernel<E4M3, GATED, 128>>(tiles * p.split, kAnyThreads, p.split, any_smem<128>(), s, p);
}

template <bool E4M3>
static collage_status_t any_forward(const collage_matrix_t* x, const collage_matrix_t* wg, const collage_matrix_t* wu, const collage_matrix_t* h,
                                    const collage_matrix_t* gate, const collage_matrix_t* up, const float* const (&scales)[3], int activation,
                                    int sm_count, cudaStream_t s) {
    AnyArgs p = {};
    p.a[0] = by_row(wg);
    p.a[1] = by_row(wu);
    p.b[0] = by_row(x);
    const collage_matrix_t* outs[3] = {h, gate, up};
    for (int i = 0; i < 3 && outs[i]; ++i) {
        p.out[i] = static_cast<uint16_t*>(outs[i]->data);
        p.ldo[i] = outs[i]->ld;
    }
    p.token_scale = scales[0];
    p.row_scale[0] = scales[1];
    p.row_scale[1] = scales[2];
    p.m = static_cast<uint32_t>(h->cols);
    p.n = static_cast<uint32_t>(h->rows);
    p.k = static_cast<uint32_t>(x->cols);
    p.terms = 1;
    p.keep = gate != nullptr;
    p.activation = activation;
    return launch_any<E4M3, true>(p, sm_count, s);
}

// out[t, i] = sum over terms and k of a[i, k] b[t, k]
static collage_status_t any_product(const Operand (&a)[2], const Operand (&b)[2], uint32_t terms, uint64_t k, const collage_matrix_t* out,
                                    int sm_count, cudaStream_t s) {
    AnyArgs p = {};
    for (uint32_t i = 0; i < terms; ++i) {
        p.a[i] = a[i];
        p.b[i] = b[i];
    }
    p.out[0] = static_cast<uint16_t*>(out->data);
    p.ldo[0] = out->ld;
    p.m = static_cast<uint32_t>(out->cols);
    p.n = static_cast<uint32_t>(out->rows);
    p.k = static_cast<uint32_t>(k);
    p.terms = terms;
    return launch_any<false, false>(p, sm_count, s);
}

static bool known(collage_activation_t a) { return a == COLLAGE_ACT_SILU || a == COLLAGE_ACT_GELU_TANH; }

// Shapes of x [tokens, width], two weights [ffn, width] and an output [tokens, ffn]
static bool shapes_fit(const collage_matrix_t* x, const collage_matrix_t* wg, const collage_matrix_t* wu, const collage_matrix_t* h) {
    return same_shape(wg, wu) && x->cols == wg->cols && h->rows == x->rows && h->cols == wg->rows;
}

template <int N>
static collage_status_t check_all(const collage_matrix_t* const (&m)[N], uint32_t elem_bytes) {
    for (const collage_matrix_t* x : m)
        if (x)
            if (const collage_status_t st = check_matrix(x, elem_bytes); st != COLLAGE_OK) return st;
    return COLLAGE_OK;
}

}  // namespace ops
}  // namespace collage

using namespace collage;
using namespace collage::ops;

extern "C" {

collage_status_t collage_gated_ffn(const collage_matrix_t* x, const collage_matrix_t* w_gate, const collage_matrix_t* w_up,
                                   const collage_matrix_t* h, const collage_matrix_t* gate, const collage_matrix_t* up,
                                   collage_activation_t activation, void* stream) {
    if (!x || !w_gate || !w_up || !h || !gate != !up) return COLLAGE_ERR_NULL;
    if (!known(activation) || !shapes_fit(x, w_gate, w_up, h)) return COLLAGE_ERR_ARG;
    if (gate && !(same_shape(gate, h) && same_shape(up, h))) return COLLAGE_ERR_ARG;
    const collage_matrix_t* all[6] = {x, w_gate, w_up, h, gate, up};
    collage_status_t st = check_all(all, 2);
    if (st != COLLAGE_OK) return st;
    AliasCheck alias;
    for (int i = 0; i < 6; ++i)
        if (all[i]) alias.add(span_of(all[i], 2), i >= 3);
    if (alias.clash()) return COLLAGE_ERR_ALIAS;
    DeviceInfo dev;
    if ((st = current_device(&dev)) != COLLAGE_OK) return st;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (h->rows == 0 || h->cols == 0) return COLLAGE_OK;
    if (x->cols == 0) {                                    // sums over no terms: gate = up = 0, h = a(0) * 0
        for (int i = 3; i < 6 && st == COLLAGE_OK; ++i)
            if (all[i]) st = clear_matrix(all[i], 2, s);
        return st;
    }
    bool maps = true;
    for (const collage_matrix_t* m : all) maps = maps && (!m || mappable(m, 2));
    if (maps) return tiles_forward<false>(x, w_gate, w_up, h, gate, up, {nullptr, nullptr, nullptr}, activation, dev.sm_count, s);
    return any_forward<false>(x, w_gate, w_up, h, gate, up, {nullptr, nullptr, nullptr}, activation, dev.sm_count, s);
}

collage_status_t collage_gated_ffn_e4m3(const collage_matrix_t* x8, const float* x_scale, const collage_matrix_t* w_gate8,
                                        const float* w_gate_scale, const collage_matrix_t* w_up8, const float* w_up_scale,
                                        const collage_matrix_t* h, collage_activation_t activation, void* stream) {
    if (!x8 || !w_gate8 || !w_up8 || !h) return COLLAGE_ERR_NULL;
    if ((!x_scale && x8->rows) || (!w_gate_scale && w_gate8->rows) || (!w_up_scale && w_up8->rows)) return COLLAGE_ERR_NULL;
    if (!known(activation) || !shapes_fit(x8, w_gate8, w_up8, h)) return COLLAGE_ERR_ARG;
    const collage_matrix_t* in[3] = {x8, w_gate8, w_up8};
    const float* scales[3] = {x_scale, w_gate_scale, w_up_scale};
    collage_status_t st = check_all(in, 1);
    if (st == COLLAGE_OK) st = check_matrix(h, 2);
    if (st != COLLAGE_OK) return st;
    AliasCheck alias;
    for (int i = 0; i < 3; ++i) {
        if (reinterpret_cast<uintptr_t>(scales[i]) % 4) return COLLAGE_ERR_ARG;
        alias.add(span_of(in[i], 1), false);
        alias.add(span_of(scales[i], 4 * in[i]->rows), false);
    }
    alias.add(span_of(h, 2), true);
    if (alias.clash()) return COLLAGE_ERR_ALIAS;
    DeviceInfo dev;
    if ((st = current_device(&dev)) != COLLAGE_OK) return st;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (h->rows == 0 || h->cols == 0) return COLLAGE_OK;
    if (x8->cols == 0) return clear_matrix(h, 2, s);
    if (mappable(x8, 1) && mappable(w_gate8, 1) && mappable(w_up8, 1) && mappable(h, 2))
        return tiles_forward<true>(x8, w_gate8, w_up8, h, nullptr, nullptr, {x_scale, w_gate_scale, w_up_scale}, activation, dev.sm_count, s);
    return any_forward<true>(x8, w_gate8, w_up8, h, nullptr, nullptr, {x_scale, w_gate_scale, w_up_scale}, activation, dev.sm_count, s);
}

collage_status_t collage_gated_ffn_backward(const collage_matrix_t* dh, const collage_matrix_t* x, const collage_matrix_t* w_gate,
                                            const collage_matrix_t* w_up, const collage_matrix_t* gate, const collage_matrix_t* up,
                                            const collage_matrix_t* dgate, const collage_matrix_t* dup, const collage_matrix_t* dx,
                                            const collage_matrix_t* dw_gate, const collage_matrix_t* dw_up,
                                            collage_activation_t activation, void* stream) {
    if (!dh || !gate || !up || !dgate || !dup || !dw_gate != !dw_up) return COLLAGE_ERR_NULL;
    if ((dx && (!w_gate || !w_up)) || (dw_gate && !x)) return COLLAGE_ERR_NULL;
    if (!known(activation)) return COLLAGE_ERR_ARG;
    if (!same_shape(gate, dh) || !same_shape(up, dh) || !same_shape(dgate, dh) || !same_shape(dup, dh)) return COLLAGE_ERR_ARG;
    if (dx && !shapes_fit(dx, w_gate, w_up, dh)) return COLLAGE_ERR_ARG;
    if (dw_gate && !shapes_fit(x, dw_gate, dw_up, dh)) return COLLAGE_ERR_ARG;
    if (!dx) w_gate = w_up = nullptr;                      // not used
    if (!dw_gate) x = nullptr;
    const collage_matrix_t* all[11] = {dh, x, w_gate, w_up, gate, up, dgate, dup, dx, dw_gate, dw_up};
    collage_status_t st = check_all(all, 2);
    if (st != COLLAGE_OK) return st;
    AliasCheck alias;
    int at[11];
    for (int i = 0; i < 11; ++i) at[i] = all[i] ? alias.add(span_of(all[i], 2), i >= 6) : -1;
    const int pairs[2][2] = {{at[4], at[6]}, {at[5], at[7]}};
    if (alias.clash(pairs)) return COLLAGE_ERR_ALIAS;
    DeviceInfo dev;
    if ((st = current_device(&dev)) != COLLAGE_OK) return st;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (dh->rows && dh->cols) {
        GateArgs g = {};
        g.dh = static_cast<const uint16_t*>(dh->data);
        g.gate = static_cast<const uint16_t*>(gate->data);
        g.up = static_cast<const uint16_t*>(up->data);
        g.dgate = static_cast<uint16_t*>(dgate->data);
        g.dup = static_cast<uint16_t*>(dup->data);
        g.lddh = dh->ld;
        g.ldg = gate->ld;
        g.ldu = up->ld;
        g.lddg = dgate->ld;
        g.lddu = dup->ld;
        g.cols = dh->cols;
        g.activation = activation;
        bool vectors = dh->cols % 8 == 0;
        for (const collage_matrix_t* m : {dh, gate, up, dgate, dup}) vectors = vectors && rows_aligned(m, 2, 16);
        const uint64_t blocks = (dh->rows * (dh->cols / 8) + 255) / 256;
        st = vectors ? launch<&gate_backward_kernel>(std::min<uint64_t>(blocks, 8ull * dev.sm_count), 256, 1, 0, s, g, dh->rows)
                     : launch<&gate_backward_any_kernel>(dh->rows, 256, 1, 0, s, g);
        if (st != COLLAGE_OK) return st;
    }
    // a product over no tokens or no channels is zero
    if (dh->rows == 0 || dh->cols == 0) {
        if (dx) st = clear_matrix(dx, 2, s);
        if (dw_gate && st == COLLAGE_OK) st = clear_matrix(dw_gate, 2, s);
        if (dw_gate && st == COLLAGE_OK) st = clear_matrix(dw_up, 2, s);
        return st;
    }
    const bool maps = mappable(dgate, 2) && mappable(dup, 2);
    const bool dx_maps = dx && dx->cols && maps && mappable(dx, 2) && mappable(w_gate, 2) && mappable(w_up, 2);
    const bool dw_maps = dw_gate && x->cols && maps && mappable(x, 2) && mappable(dw_gate, 2) && mappable(dw_up, 2);
    if (dx_maps && dw_maps && slim_dx(dx, dev.sm_count) && small_layer(dh->rows, dw_gate, dev.sm_count))
        return slim_backward(dgate, dup, x, w_gate, w_up, dx, dw_gate, dw_up, dev.sm_count, s);
    if (dx_maps) {
        if ((st = tiles_dx(dgate, dup, w_gate, w_up, dx, dev.sm_count, s)) != COLLAGE_OK) return st;
        dx = nullptr;
    }
    if (dw_maps) {
        if ((st = tiles_dw(dgate, dup, x, dw_gate, dw_up, dev.sm_count, s)) != COLLAGE_OK) return st;
        dw_gate = nullptr;
    }
    if (dx && dx->cols)
        if ((st = any_product({by_col(w_gate), by_col(w_up)}, {by_row(dgate), by_row(dup)}, 2, dh->cols, dx, dev.sm_count, s)) != COLLAGE_OK) return st;
    for (int half = 0; half < 2 && dw_gate && x->cols; ++half)
        if ((st = any_product({by_col(x), {}}, {by_col(half ? dup : dgate), {}}, 1, dh->rows, half ? dw_up : dw_gate, dev.sm_count, s)) != COLLAGE_OK) return st;
    return COLLAGE_OK;
}

}  // extern "C"

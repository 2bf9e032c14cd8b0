/*
 * collage.h -- C ABI of the B200 (sm_100a) Collage bf16 multi-component-float AdamW library.
 *
 * The library implements the optimizer step of "Collage: Light-Weight Low-Precision Strategy
 * for LLM Training" (Algorithm 2) for the paper's precision options A (plain bfloat16),
 * B (Collage-light: theta held as a bfloat16 pair) and C (Collage-plus: theta and the second
 * moment held as pairs, beta2 as a pair), the error-free transforms it is built from
 * (Theorem 4.1, Algorithm 1, Appendix C), and the effective-descent-quality metric (Eq. 2-3).
 *
 * Arithmetic model (Section 3.1): every operator written in the paper takes bfloat16 operands
 * and rounds its exact result once, to nearest-even, to bfloat16.  Scalars are evaluated in
 * double on the host and cast to bfloat16 last (Section 4.2, Appendix D).
 *
 * Conventions for every entry point unless it says otherwise:
 *   - tensor pointers are DEVICE pointers to bfloat16 bit patterns (uint16_t), owned by the
 *     caller, on the current CUDA device; hyper-parameter structs, tensor lists and scalar
 *     outputs named "host" are HOST pointers;
 *   - state tensors are updated in place; `grad` is read only;
 *   - calls are asynchronous on `stream` (a cudaStream_t passed as void*; NULL = default
 *     stream); the library never synchronises the device and never allocates on the step path;
 *     collage_adamw_step, collage_adamw_step_multi and collage_adamw_step_fp32 only launch kernels,
 *     so once a call of the same kind has run on the device (it sets per-device kernel attributes
 *     the first time) they may be recorded by stream capture into a CUDA graph: the scalars of
 *     the step are kernel arguments and are recorded with it;
 *   - errors are detected on the host BEFORE anything is launched and reported as a status
 *     code; nothing is thrown across the boundary; there is no CPU fallback: a device that is
 *     not compute capability 10.x yields COLLAGE_ERR_ARCH;
 *   - pointers need not be 16-byte aligned and lengths need not be multiples of 8 (such
 *     tensors take a slower element-wise path with identical results);
 *   - n == 0 is a successful no-op;
 *   - NaN/Inf in tensor data is not an error: it propagates per IEEE 754;
 *   - threads: any entry point may be called from several host threads at once, on the same or on
 *     different devices and streams (the library's own first-call set-up is guarded), provided that
 *     calls in flight together share no tensor, no workspace, no plan being modified
 *     (collage_plan_set_replicas, collage_plan_destroy) and, for collage_adamw_step_host and
 *     collage_edq_static, no device: those two keep one context or scratch array per device;
 *   - the EDQ workspace (hyper->workspace) must hold zeros before its first use: clear it once with
 *     collage_workspace_init or cudaMemset.  Every call leaves it ready for the next one.
 */
#ifndef COLLAGE_H_
#define COLLAGE_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    COLLAGE_OK = 0,
    COLLAGE_ERR_NULL = 1,       /* a required pointer is NULL                                   */
    COLLAGE_ERR_ARG = 2,        /* step == 0, unknown strategy/op/flag combination, hyper out of range */
    COLLAGE_ERR_ALIAS = 3,      /* two tensors of one call overlap, or one overlaps the workspace / EDQ record */
    COLLAGE_ERR_ARCH = 4,       /* current device is not sm_100                                 */
    COLLAGE_ERR_CUDA = 5,       /* a CUDA runtime call or launch failed                         */
    COLLAGE_ERR_WORKSPACE = 6,  /* workspace missing or smaller than collage_workspace_bytes()  */
    COLLAGE_ERR_LIMIT = 7       /* size beyond the fixed capacity of an entry point             */
} collage_status_t;

/* Precision options of Table 2. */
typedef enum {
    COLLAGE_BF16 = 0,   /* A: theta, m, v single bfloat16                    ( 8 B/param with grad) */
    COLLAGE_LIGHT = 1,  /* B: (theta, dtheta) pair                           (10 B/param)           */
    COLLAGE_PLUS = 2,   /* C: (theta, dtheta), (v, dv) pairs, beta2 as pair  (12 B/param)           */
    /* Comparator of the paper's experiments, not one of its options: BF16 AdamW with Kahan summation
     * at the parameter update (Appendix B): update' = update (+) c; theta' = theta (+) update';
     * c' = update' (-) (theta' (-) theta).  Same arrays as option B, x_lo holding c (10 B/param).
     * EDQ counts theta alone (Eq. 2 as printed). */
    COLLAGE_KAHAN = 3,
    /* A measuring stick outside the paper (its Algorithm 2 is strict bfloat16): option C's arrays and
     * traffic, but each step widens theta+dtheta and v+dv to float, runs AdamW in IEEE single
     * operations with float scalars, and splits the results back into normalised bfloat16 pairs
     * (hi = RN(x), lo = RN(x - hi)).  Quantifies what the strict arithmetic costs in accuracy. */
    COLLAGE_PLUS_FP32_REGISTERS = 4
} collage_strategy_t;

/* Algorithm 2 line 12 prints epsilon under the root; AdamW has it outside.  Default: outside. */
#define COLLAGE_FLAG_EPS_INSIDE_SQRT 1u
/* Variants of the parameter update (default: off).
 * TWOSUM_GROW: line 13's Grow uses TwoSum instead of Fast2Sum (Appendix C: same expansion with no
 *   ordering requirement), so the update is error-free also where |theta| < |update|.  B and C only.
 * DECAY_BY_GROW: the weight decay is not summed into the update (Appendix D: "either ... or") but
 *   applied first by an addition (Grow for B and C) of its own: d = (-a) (*) (lam (*) theta), then the
 *   Adam part (-a) (*) r.  A, B, C.  EDQ then measures against d + update. */
#define COLLAGE_FLAG_TWOSUM_GROW 2u
#define COLLAGE_FLAG_DECAY_BY_GROW 4u
/* Which kernel runs the step.  By default the size decides: a flat tensor of up to 2^21 parameters takes
 * a kernel without staging, one 8-parameter vector per thread straight from global memory (shortest
 * latency); above that, and for every multi-tensor plan, the bulk-copy pipeline streams at HBM bandwidth
 * in three stages of 4096-element tiles (6144 for COLLAGE_BF16); a COLLAGE_PLUS step over 2^27 parameters or
 * more uses two stages of 8192-element tiles (1-2 % faster there; in a plan only if chunk_elems is a
 * multiple of 8192, as the default is).  All of them compute the same bits.  These flags pin the choice
 * (tests and measurements): PIPELINE_KERNEL = the three-stage pipeline whatever the size, DIRECT_KERNEL =
 * the kernel without staging (flat entry points only), LARGE_TILES = the two-stage pipeline (COLLAGE_PLUS
 * without variant flags only).  More than one of them is ERR_ARG; where a flag does not apply it is ignored. */
#define COLLAGE_FLAG_PIPELINE_KERNEL 8u
#define COLLAGE_FLAG_DIRECT_KERNEL 16u
#define COLLAGE_FLAG_LARGE_TILES 32u

/* Hyper-parameters of one step (Algorithm 2 line 1).  HOST struct.
 * Valid ranges: lr, eps, weight_decay >= 0 and finite; 0 <= beta1, beta2 < 1. */
typedef struct collage_hyper {
    double lr, beta1, beta2, eps, weight_decay;
    uint32_t flags;          /* COLLAGE_FLAG_*                                                   */
    void* edq_out;           /* DEVICE collage_edq_t*, or NULL to skip the EDQ reduction          */
    void* workspace;         /* DEVICE scratch, >= collage_workspace_bytes(); needed iff edq_out  */
    size_t workspace_bytes;
} collage_hyper_t;

/* Result of the EDQ reduction (Eq. 3), written on the device by the call's last kernel.
 *   dot   = sum_i delta_i * eff_i        eff = (theta'+dtheta') - (theta+dtheta)   (Eq. 2)
 *   sumsq = sum_i delta_i^2              delta = the bfloat16 update of Algorithm 2 line 12
 *   edq   = dot / sqrt(sumsq), 0 if sumsq == 0
 *   lost  = #{i : delta_i != 0 and eff_i == 0}: parameters that an update was meant for and that did not
 *           move (Def. 3.2; "not updated", Figure 3 left).  For a pair the value theta + dtheta counts:
 *           a Grow that re-splits the same value over other components has not updated it.
 *   fault = 0, or the code of a bounded device-side wait that gave up during this call (see
 *           collage_pipeline_fault): the step was torn and the state arrays are then undefined.
 * Products and 8-element partial sums are formed in float, everything above in double, in a
 * fixed order: the result is reproducible for a given launch geometry. */
typedef struct collage_edq {
    double dot, sumsq, edq;
    uint64_t n;
    uint64_t lost;
    uint64_t fault;
} collage_edq_t;

/* One parameter tensor of a multi-tensor plan.  x_lo may be NULL for a plan used only with
 * COLLAGE_BF16; v_lo may be NULL unless the plan is used with COLLAGE_PLUS. */
typedef struct collage_tensor {
    void* x_hi;        /* theta          */
    void* x_lo;        /* delta-theta    */
    void* m;           /* first moment   */
    void* v_hi;        /* second moment  */
    void* v_lo;        /* delta-v        */
    const void* grad;
    uint64_t n;        /* elements       */
} collage_tensor_t;

typedef struct collage_plan collage_plan_t;   /* opaque; owns a small device table */

const char* collage_status_string(collage_status_t status);

/* Scalar preparation (Algorithm 2 line 1; Table 1; Appendix D "Scalar and Bias Correction").
 * HOST only, no CUDA call.  out_bf16[11] receives, as bfloat16 bit patterns,
 *   [0] RN(beta1) [1] RN(1-beta1) [2] RN(beta2) [3] RN(1-beta2)
 *   [4] beta2_hi = RN(beta2) [5] beta2_lo = RN(beta2 - beta2_hi)
 *   [6] RN(1-beta1^step) [7] RN(1-beta2^step) [8] RN(lr) [9] RN(weight_decay) [10] RN(eps)
 * every expression evaluated in double before the one rounding.
 * Errors: NULL -> ERR_NULL; step == 0 or hyper out of range -> ERR_ARG. */
collage_status_t collage_derive_scalars(const collage_hyper_t* hyper, uint64_t step, uint16_t out_bf16[11]);

/* Bytes of device scratch the EDQ reduction needs (independent of n; about 128 KiB). */
size_t collage_workspace_bytes(uint64_t n_total);

/* Clears an EDQ workspace (asynchronous memset on `stream`).  The step kernels end their EDQ
 * reduction (Eq. 3) inside the same launch: each thread block stores its partial sums in the
 * workspace and draws a ticket from a counter that lives there; the block that draws the last
 * ticket adds the partials in index order and writes the record.  The counter wraps back to zero
 * with the last ticket, so one clearing before the first use is enough.  A workspace serves one
 * call at a time: calls that may run concurrently need separate workspaces.
 * Errors: ERR_NULL, ERR_WORKSPACE (smaller than collage_workspace_bytes() or not 16-byte aligned),
 * ERR_CUDA. */
collage_status_t collage_workspace_init(void* workspace, size_t workspace_bytes, void* stream);

/* Combines EDQ records of disjoint parameter sets (tensors, slices, ranks) into the record of their
 * union, Eq. 3 on the summed partial sums: dot, sumsq, n and lost are added in array order, edq =
 * dot / sqrt(sumsq) (0 if sumsq == 0), fault = the first non-zero fault.  HOST arrays, no CUDA call.
 * `out` may be one of the parts.  Errors: ERR_NULL, ERR_ARG (count < 0). */
collage_status_t collage_edq_combine(const collage_edq_t* parts_host, int count, collage_edq_t* out_host);

/* "product" for the ordinary build; a measurement build of the same sources that compiles the
 * arithmetic out of the step kernel (to time the copy pipeline alone) answers "data-movement-only". */
const char* collage_build_flavor(void);

/* One AdamW step over one flat tensor (Algorithm 2 lines 8-13, all n parameters, step t >= 1).
 *   x_hi, m, v_hi, grad : required.   x_lo : required iff strategy != COLLAGE_BF16 (delta-theta, or
 *   the Kahan compensation for COLLAGE_KAHAN), else must
 *   be NULL.   v_lo : required iff strategy is COLLAGE_PLUS or COLLAGE_PLUS_FP32_REGISTERS, else
 *   must be NULL.
 * With hyper->edq_out set the record is written by the same launch (one kernel per step).
 * Errors: ERR_NULL, ERR_ARG (step 0, bad strategy, hyper range), ERR_ALIAS (overlapping
 * tensors; workspace or record overlapping a tensor or each other), ERR_WORKSPACE (edq_out set,
 * workspace missing, misaligned or too small), ERR_ARCH, ERR_CUDA. */
collage_status_t collage_adamw_step(void* x_hi, void* x_lo, void* m, void* v_hi, void* v_lo,
                                    const void* grad, uint64_t n, const collage_hyper_t* hyper,
                                    uint64_t step, collage_strategy_t strategy, void* stream);

/* Comparator of the paper's experiments: option D of Table 2 -- bfloat16 parameter and gradient,
 * float (fp32) optimizer states and float master weights, 16 B/param -- and, with master == NULL,
 * D^-MW of Section 5.1 (float optimizer states, no master weights, 12 B/param).  Standard
 * mixed-precision AdamW in the operation order of Algorithm 2; every operation is one IEEE
 * single-precision operation, scalars are evaluated in double and cast to float once.
 *   theta : DEVICE bfloat16[n], written (D: theta = RN_bf16(master); D^-MW: read and written)
 *   master: DEVICE float[n] or NULL;  m, v: DEVICE float[n];  grad: DEVICE bfloat16[n], read only
 * EDQ (hyper->edq_out / workspace as for collage_adamw_step) measures the float update against the
 * change of the stored parameter: the master weight for D, the bfloat16 parameter for D^-MW.
 * HBM traffic 28 B/param (D) or 22 B/param (D^-MW) against 22 B/param of Collage-plus.
 * Of the arithmetic flags only COLLAGE_FLAG_EPS_INSIDE_SQRT is accepted in hyper->flags.
 * Errors: ERR_NULL, ERR_ARG (step 0, hyper range, flags, float arrays not 4-byte aligned),
 * ERR_ALIAS, ERR_WORKSPACE, ERR_ARCH, ERR_CUDA. */
collage_status_t collage_adamw_step_fp32(void* theta, void* master, void* m, void* v, const void* grad,
                                         uint64_t n, const collage_hyper_t* hyper, uint64_t step, void* stream);

/* The same step for state that lives in HOST memory (optimizer state kept off the device).
 * All six tensor pointers are HOST pointers (page-locked memory is needed for the copies to
 * overlap; pageable memory works, serialised by the runtime).  The arrays are streamed through
 * `staging_dev`, a DEVICE buffer of `staging_bytes` bytes (256-byte aligned, at least
 * collage_workspace_bytes() + 1 MiB; larger is faster up to a few hundred MiB), in slabs: while
 * slab i is computed, slab i+1 is copied in and slab i-1 copied out on two internal copy streams
 * that the library creates per device on the first call.  Work is ordered after earlier work on
 * `stream`, and `stream` waits for the last copy-out, so synchronising `stream` suffices.
 * hyper->edq_out, if set, is a HOST collage_edq_t* here (written by a copy enqueued on
 * `stream`); hyper->workspace is ignored.  Results are bit-identical to collage_adamw_step.
 * Calls on one device share the copy streams: issue them one at a time per device.
 * Errors: as collage_adamw_step, with ERR_WORKSPACE for a missing, misaligned or too small
 * staging buffer. */
collage_status_t collage_adamw_step_host(void* x_hi, void* x_lo, void* m, void* v_hi, void* v_lo,
                                         const void* grad, uint64_t n, const collage_hyper_t* hyper,
                                         uint64_t step, collage_strategy_t strategy, void* staging_dev,
                                         size_t staging_bytes, void* stream);

/* Multi-tensor step: all tensors of a plan in ONE launch over a chunk table.
 * collage_plan_create copies the HOST array `tensors[num]` and builds the device table
 * (this call allocates and synchronises; do it once, outside the step loop).  chunk_elems is
 * the work unit handed to a thread block, a multiple of 2048; 0 picks the default (24576;
 * multiples of 24576 keep every tile whole for every precision option and tile size).
 * Tensors with n == 0 are skipped.  The plan records which pointers were NULL; a step whose
 * strategy needs a missing component fails with ERR_NULL.  EDQ is over all tensors (Eq. 3
 * with theta the concatenation).
 * A plan belongs to the device that was current at creation; stepping it with another device
 * current is ERR_ARG.
 * Errors: ERR_NULL, ERR_ARG (num < 0, chunk_elems not a multiple of 2048, more than 2^32-1
 * chunks), ERR_ALIAS (any two arrays of the plan overlap), ERR_CUDA. */
collage_status_t collage_plan_create(const collage_tensor_t* tensors, int num, uint32_t chunk_elems,
                                     collage_plan_t** out_plan);
collage_status_t collage_adamw_step_multi(const collage_plan_t* plan, const collage_hyper_t* hyper,
                                          uint64_t step, collage_strategy_t strategy, void* stream);
collage_status_t collage_plan_destroy(collage_plan_t* plan);

/* Replicas of the parameter (sharded optimizer state: each GPU steps its own slice of the
 * parameters, every GPU needs all of theta for the next forward pass).  After this call every
 * step of the plan also writes the updated first component theta of tensor i to each replica,
 * tile by tile from inside the step kernel (the same bulk stores that write theta home), so the
 * gather costs no extra kernel and overlaps the step.  The paper describes no collective; this is
 * the one exchange its optimizer step would need (2 B/param per replica).
 *   replicas : HOST array of num_replicas * num DEVICE pointers, replica r of tensors[i] at
 *              replicas[r * num + i], `num` as given to collage_plan_create; each points to
 *              tensors[i].n bfloat16 values in this GPU's memory or in a peer GPU's memory mapped
 *              into this process (peer access enabled), and must have the same address modulo 16
 *              as tensors[i].x_hi.  Entries of empty tensors are ignored.  num_replicas <= 15;
 *              0 removes the replicas.
 * The call synchronises the device and allocates a small table: do it once, outside the step loop.
 * A replica holds the new theta once the step's kernel has finished; readers on other GPUs need
 * their own ordering with that (an event, a barrier).  Plain stores issued by each block for itself.
 * Errors: ERR_NULL, ERR_ARG (count, alignment, wrong device), ERR_ALIAS (a replica overlaps an
 * array of the plan or another replica), ERR_CUDA. */
collage_status_t collage_plan_set_replicas(collage_plan_t* plan, const void* const* replicas, int num_replicas);

/* Lets kernels of the CURRENT device store into memory of `peer_device` (a device ordinal of this
 * process), so that pointers into a peer's memory that the caller has mapped (CUDA IPC, virtual
 * memory management) can serve as replicas.  Host-side set-up, not on the step path; succeeds if the
 * access is already enabled.  The paper has no counterpart (its experiments do not shard the step).
 * Errors: ERR_ARG (same device, or the devices cannot reach each other), ERR_CUDA. */
collage_status_t collage_enable_peer_access(int peer_device);

/* The multi-tensor step with EDQ kept per tensor (Eq. 2-3 evaluated on each parameter tensor of the
 * plan separately; the lost-update count of Def. 3.2 per tensor gives the imprecision percentage of
 * Figure 3, left).  Same state update as collage_adamw_step_multi, bit for bit.
 *   per_tensor_out_dev : DEVICE collage_edq_t[num], num = the `num` given to collage_plan_create;
 *                        entry i belongs to tensors[i] (all zero for an empty tensor).
 *   chunk_workspace    : DEVICE scratch of at least collage_plan_workspace_bytes(plan) bytes, 16-byte
 *                        aligned (32 bytes per chunk of the plan).
 *   hyper->edq_out     : optional DEVICE collage_edq_t for the whole plan = the per-tensor sums added
 *                        in tensor order (association differs from collage_adamw_step_multi's, so
 *                        the last bits may differ); hyper->workspace is not used by this call.
 * Three launches (step, per-tensor sums, total) instead of one.  The variant flags (TWOSUM_GROW,
 * DECAY_BY_GROW) are not available through this entry point (ERR_ARG).
 * Errors: as collage_adamw_step_multi, plus ERR_ARG when num differs from the plan's and
 * ERR_WORKSPACE for the chunk workspace. */
size_t collage_plan_workspace_bytes(const collage_plan_t* plan);
collage_status_t collage_adamw_step_multi_per_tensor(const collage_plan_t* plan, const collage_hyper_t* hyper,
                                                     uint64_t step, collage_strategy_t strategy,
                                                     collage_edq_t* per_tensor_out_dev, int num,
                                                     void* chunk_workspace, size_t chunk_workspace_bytes,
                                                     void* stream);
/* Plan facts for callers that report or shard: total elements, number of chunks. */
uint64_t collage_plan_num_elements(const collage_plan_t* plan);
uint64_t collage_plan_num_chunks(const collage_plan_t* plan);

/* Batched MCF primitives, elementwise over n bfloat16 values.  Output arrays may be the input
 * arrays themselves (exact same pointer); partial overlap is ERR_ALIAS.
 *   fast_two_sum (Theorem 4.1): hi = a (+) b, lo = b (-) (hi (-) a); error-free if |a| >= |b|
 *   two_sum      (Algorithm TwoSum): same expansion, no ordering needed, 6 operations
 *   two_prod     (Algorithm TwoProdFMA): hi = a (*) b, lo = fma(a, b, -hi)
 *   grow         (Algorithm 1): (u, v) = Fast2Sum(x, a); (u, v) = Fast2Sum(u, y (+) v)
 *   scaling      (Algorithm Scaling): float v times expansion (a1, a2)
 *   mul          (Algorithm Mul): expansion (a1, a2) times expansion (b1, b2)
 *   renormalize  (named in the paper's listing keywords, not defined there): Fast2Sum(hi, lo) */
collage_status_t collage_fast_two_sum(const void* a, const void* b, void* hi, void* lo, uint64_t n, void* stream);
collage_status_t collage_two_sum(const void* a, const void* b, void* hi, void* lo, uint64_t n, void* stream);
collage_status_t collage_two_prod(const void* a, const void* b, void* hi, void* lo, uint64_t n, void* stream);
collage_status_t collage_grow(const void* x, const void* y, const void* a, void* u, void* v, uint64_t n, void* stream);
collage_status_t collage_scaling(const void* v, const void* a1, const void* a2, void* x, void* e, uint64_t n, void* stream);
collage_status_t collage_mul(const void* a1, const void* a2, const void* b1, const void* b2, void* x, void* e,
                             uint64_t n, void* stream);
collage_status_t collage_renormalize(const void* hi_in, const void* lo_in, void* hi, void* lo, uint64_t n, void* stream);

/* One rounded bfloat16 operation F^BF16(a op b) elementwise (Section 3.1), realised exactly as
 * inside the step kernel.  op: 0 add, 1 sub, 2 mul, 3 div, 4 sqrt(a), 5 fma(a,b,c).  b is
 * ignored for sqrt; c only used by fma (pass NULL otherwise). */
collage_status_t collage_rounded_op(int op, const void* a, const void* b, const void* c, void* out,
                                    uint64_t n, void* stream);

/* EDQ on stored arrays (Eq. 2-3): old and new parameter expansions and the intended update.
 * old_lo/new_lo both NULL = plain bfloat16 parameter.  out_dev: DEVICE collage_edq_t*.
 * Errors: ERR_NULL, ERR_WORKSPACE, ERR_ARCH, ERR_CUDA. */
collage_status_t collage_edq(const void* old_hi, const void* old_lo, const void* new_hi,
                             const void* new_lo, const void* delta, uint64_t n, collage_edq_t* out_dev,
                             void* workspace, size_t workspace_bytes, void* stream);

/* EDQ for callers that cannot allocate device memory (the paper has no counterpart; this is an
 * interface convenience, the computation is collage_edq's).  Some callers own no allocator they
 * may call at this point: a training process that has handed every byte of the GPU to a memory
 * pool and forbids raw cudaMalloc inside the step (it can fail, and it synchronises the device),
 * a plugin running inside someone else's framework without access to its allocator, or code in a
 * latency-critical region.  For them the scratch that collage_edq takes as `workspace` is built
 * into the library: a fixed 64 KiB array in device memory (2048 partial sums), which every GPU
 * that loads the library holds until the process exits.  Arguments are those of collage_edq
 * without workspace; `out_dev` is still the caller's DEVICE collage_edq_t.
 *   - Capacity: the array has 2048 slots and a thread block reduces up to 2^21 elements, so
 *     n <= 2^32; a larger n is rejected with COLLAGE_ERR_LIMIT and nothing is launched.
 *   - The call itself allocates nothing and frees nothing.  The first call on each device looks up
 *     the array's device address (cudaGetSymbolAddress, with that device current); make that first
 *     call before any stream capture begins.
 *   - All calls on a device share the one array.  Each call overwrites every slot it later reads,
 *     so nothing needs clearing between calls; but two calls whose kernels overlap on the GPU
 *     (different streams, no ordering) race on it.  Order them, or use collage_edq with separate
 *     workspaces.
 *   - The sums are grouped per segment of ceil(n / 2048) elements (rounded up to a multiple of 8,
 *     at least 2048), a function of n alone and not of the launch geometry, so they can differ from
 *     collage_edq's in the last bits (same tolerance as against the CPU oracle).
 * Errors: ERR_NULL, ERR_LIMIT, ERR_ARCH, ERR_CUDA. */
collage_status_t collage_edq_static(const void* old_hi, const void* old_lo, const void* new_hi,
                                    const void* new_lo, const void* delta, uint64_t n,
                                    collage_edq_t* out_dev, void* stream);

/* The step kernel's copy pipeline waits on shared-memory barriers with a bound of two seconds of
 * the device's wall clock; a wait that runs out records a code in a device word and the block
 * leaves, so a fault can never hang the device.  The kernel still ends normally and the call has
 * long returned COLLAGE_OK, but the step was torn: the state arrays are undefined from then on.
 * A step that reduces EDQ copies the word into its record (collage_edq_t.fault), so a caller that
 * reads the record sees the fault at once.  This call copies the word to *out_host (0 = no fault
 * seen on the current device since the last read) and clears it.  It synchronises the device: call
 * it at checkpoints, not per step.  The feed-forward products below (collage_gated_ffn and its kin), the multi-tensor AdamW step
 * (collage_adam_step) and collage_block_norm_backward wait in the same way and report codes above 200, 300 and 400 here: their
 * outputs are then undefined.  Errors: ERR_NULL, ERR_CUDA. */
collage_status_t collage_pipeline_fault(uint32_t* out_host);

/* Exercises the give-up path of those waits without any fault: launches one warp that waits on a
 * barrier nothing completes, bounded by `limit_ms` milliseconds (1..1000) of the device's wall
 * clock.  The wait runs out, the kernel returns normally, and the next
 * collage_pipeline_fault reports the code 100.  The device and the library stay usable.
 * Asynchronous on `stream`.  Errors: ERR_ARG (limit out of range), ERR_ARCH, ERR_CUDA. */
collage_status_t collage_wait_timeout_selftest(uint32_t limit_ms, void* stream);

/* Exhaustive self test of the arithmetic the kernels rely on, on the current device (Section 3.1's
 * model: one rounding to nearest-even per operation).  Compares, for EVERY pair of bfloat16 bit
 * patterns (2^32 pairs; 2^16 values for the root), the realisation used in the kernels with a
 * reference built from IEEE float/double arithmetic and one conversion to bfloat16:
 *   out_host[0] add  [1] sub  [2] mul            native packed bfloat16 instructions
 *   out_host[3] div  [4] sqrt                    reciprocal / root approximations vs div.rn, sqrt.rn,
 *                                                both in the form that answers every operand and in the
 *                                                branch-free form of the step kernel (whose unflagged
 *                                                lanes must be right on all operands it admits)
 *   out_host[5] division by a scalar through a host-rounded reciprocal (divisors in (0, 1])
 * Each entry is the number of results that differ (NaNs compared as a class); all must be 0.
 * HOST output; allocates a few bytes, synchronises `stream`; takes about a second.
 * Errors: ERR_NULL, ERR_ARCH, ERR_CUDA. */
collage_status_t collage_selftest(uint64_t out_host[6], void* stream);

/* ------------------------------------------------------------------------------------------------
 * Operators of a training step's forward and backward pass, next to the optimizer step that consumes
 * their gradients: residual addition + RMS norm, rounding of rows to 8 bits, the gated feed-forward
 * projections, and distillation from a teacher's top logits.  The paper describes none of them.
 *
 * Unlike Algorithm 2 they are ordinary mixed precision: operands are bfloat16 (or e4m3 where a name says
 * so), products, sums, statistics and exponentials are held in float, and a result is rounded once, when
 * it is stored.  All sums have a fixed order: a call repeated on the same device gives the same bits.
 *
 * Matrices are described by collage_matrix_t (a HOST struct, read during the call): row-major, element
 * (i, j) at data + i * ld + j elements, ld >= cols.  Rows and columns are below 2^31 (ERR_LIMIT), offsets
 * are 64-bit.  Pointers and strides need no alignment beyond their element's; matrices whose rows all
 * begin on 16 bytes are faster.  An output may overlap another array of the call only where it says so
 * (ERR_ALIAS; two matrices that interleave by columns of a common stride, such as the halves of one
 * [rows, 2 n] buffer, do not overlap).  Inputs may overlap each other.
 * Errors common to all: ERR_NULL (a required pointer), ERR_ARG (shapes that do not fit together, ld < cols,
 * misaligned elements, values out of range), ERR_LIMIT, ERR_ALIAS, ERR_ARCH, ERR_CUDA.
 * All of them only launch kernels (and clear small arrays) on `stream` and may be recorded by stream capture.  A kernel's
 * blocks may be set up while the stream's previous kernel still runs; it touches memory only after that one's end.
 * The feed-forward products wait with a bound, as the step does: one that gives up has long returned COLLAGE_OK, and only
 * collage_pipeline_fault tells that its outputs are undefined.  Ask it where a training loop reads its losses or saves. */
typedef struct collage_matrix {
    void* data;
    uint64_t rows, cols;
    uint64_t ld;             /* elements from one row's beginning to the next one's */
} collage_matrix_t;

/* r = x + residual;  rstd_i = 1 / sqrt(mean_j r_ij^2 + eps);  y_ij = r_ij * rstd_i * weight_j.
 *   x, residual : bfloat16 [rows, cols]; residual may be NULL (r = x).
 *   weight      : DEVICE bfloat16[cols].       eps >= 0 and finite.
 *   residual_out: bfloat16 [rows, cols] or NULL: r rounded, the stream that the next layer adds to.  Only
 *                 with a residual.  y is computed from r as it was before that rounding.
 *   y           : bfloat16 [rows, cols] or NULL.
 *   y8, y8_scale: e4m3 [rows, cols] and float[rows], or both NULL: y rounded to 8 bits as by
 *                 collage_quantize_rows, y ~ y8 * y8_scale.  At least one of y and y8 is given.
 *   rstd        : DEVICE float[rows] or NULL (the backward pass needs it).  NaN in rows of no columns.
 * residual_out may be the array of x or of residual, y that of x (same data, same ld).
 * A row that holds a NaN gives NaNs; one that holds an infinity has rstd 0, NaN where the infinity is and zeros elsewhere
 * (IEEE arithmetic).  Squares are held to a float's precision whatever their size: finite rows may have values up to the
 * type's largest, and with eps = 0 any rows of which 1 / rms is a float. */
collage_status_t collage_add_rms_norm(const collage_matrix_t* x, const collage_matrix_t* residual, const void* weight,
                                      double eps, const collage_matrix_t* residual_out, const collage_matrix_t* y,
                                      const collage_matrix_t* y8, float* y8_scale, float* rstd, void* stream);

/* Its backward pass.  With n = r * rstd and g = weight * dy:
 *   dx = rstd * (g - n * mean_j(g n)) + dresidual      (the gradient of x and of residual alike)
 *   dweight_j = sum_i dy_ij * n_ij
 *   dy          : bfloat16 [rows, cols], gradient of y.   r: residual_out of the forward call (x without a
 *                 residual).   rstd: of the forward call.
 *   dresidual   : bfloat16 [rows, cols] or NULL: gradient that reached residual_out on its own way.
 *   dx          : bfloat16 [rows, cols] or NULL; may be the array of dy or of dresidual.
 *   dweight     : DEVICE bfloat16[cols] or NULL (zeros if rows == 0).  One of dx and dweight is given.
 *   workspace   : DEVICE scratch of at least collage_rms_norm_workspace_bytes(cols), 16-byte aligned, needed
 *                 with dweight; nothing in it is kept between calls (ERR_WORKSPACE).
 * A gradient of 8-bit outputs passes straight through: dy is the gradient of y8 * y8_scale. */
size_t collage_rms_norm_workspace_bytes(uint64_t cols);
collage_status_t collage_add_rms_norm_backward(const collage_matrix_t* dy, const collage_matrix_t* r, const float* rstd,
                                               const void* weight, const collage_matrix_t* dresidual,
                                               const collage_matrix_t* dx, void* dweight, void* workspace,
                                               size_t workspace_bytes, void* stream);

/* One scale a row: scale_i = max_j |x_ij| / 448, q_ij = e4m3(x_ij / scale_i), to nearest even.  A row of zeros
 * has scale 0 and zeros.  A row with a NaN or an infinity has that as its scale (NaN before infinity), and q
 * follows by IEEE division: NaN where x_ij is NaN or infinite, so that q * scale is NaN in all of the row.
 *   x: bfloat16 [rows, cols];  q: e4m3 [rows, cols], one byte each;  scale: DEVICE float[rows]. */
collage_status_t collage_quantize_rows(const collage_matrix_t* x, const collage_matrix_t* q, float* scale, void* stream);

typedef enum {
    COLLAGE_ACT_SILU = 0,        /* a(g) = g / (1 + exp(-g))                                                  */
    COLLAGE_ACT_GELU_TANH = 1    /* a(g) = g / 2 * (1 + tanh(sqrt(2/pi) * (g + 0.044715 g^3)))                 */
} collage_activation_t;

/* Gated feed-forward projections: gate = x w_gate^T, up = x w_up^T, h = a(gate) * up, in one kernel.
 *   x: bfloat16 [tokens, width];  w_gate, w_up: bfloat16 [ffn, width];  h: bfloat16 [tokens, ffn].
 *   gate, up: bfloat16 [tokens, ffn], or both NULL: kept for the backward pass, in the type and size in which a
 *   training program keeps activations; the gradients carry that rounding (2^-9 of each on average, as that of dgate and
 *   dup, which the matrix instructions take in bfloat16).  h is computed from the float products, before these are rounded.
 * Widths of whole 16 bytes (8 elements; 16 of 8 bits) and rows on 16 bytes take tensor-map copies; others are
 * brought to the tensor cores element by element, about nine times slower at large sizes. */
collage_status_t collage_gated_ffn(const collage_matrix_t* x, const collage_matrix_t* w_gate, const collage_matrix_t* w_up,
                                   const collage_matrix_t* h, const collage_matrix_t* gate, const collage_matrix_t* up,
                                   collage_activation_t activation, void* stream);

/* Its backward pass: dgate = dh * up * a'(gate), dup = dh * a(gate), rounded to bfloat16, then
 *   dx = dgate w_gate + dup w_up,   dw_gate = dgate^T x,   dw_up = dup^T x.
 *   dh: bfloat16 [tokens, ffn];  x, w_gate, w_up, gate, up: of the forward call.
 *   dgate, dup: bfloat16 [tokens, ffn], written; they may be the arrays of gate and up (in that order).
 *   dx: bfloat16 [tokens, width] or NULL (w_gate and w_up are then not used and may be NULL).
 *   dw_gate, dw_up: bfloat16 [ffn, width], or both NULL (x is then not used and may be NULL). */
collage_status_t collage_gated_ffn_backward(const collage_matrix_t* dh, const collage_matrix_t* x,
                                            const collage_matrix_t* w_gate, const collage_matrix_t* w_up,
                                            const collage_matrix_t* gate, const collage_matrix_t* up,
                                            const collage_matrix_t* dgate, const collage_matrix_t* dup,
                                            const collage_matrix_t* dx, const collage_matrix_t* dw_gate,
                                            const collage_matrix_t* dw_up, collage_activation_t activation, void* stream);

/* The projections with 8-bit operands: gate_tf = x_scale_t * w_gate_scale_f * sum_d x8_td w_gate8_fd, up likewise;
 * h = a(gate) * up in bfloat16.  x8 [tokens, width], w_gate8, w_up8 [ffn, width] are e4m3; the scales are DEVICE
 * float[tokens], float[ffn], float[ffn], as collage_add_rms_norm and collage_quantize_rows write them. */
collage_status_t collage_gated_ffn_e4m3(const collage_matrix_t* x8, const float* x_scale, const collage_matrix_t* w_gate8,
                                        const float* w_gate_scale, const collage_matrix_t* w_up8, const float* w_up_scale,
                                        const collage_matrix_t* h, collage_activation_t activation, void* stream);

/* Distillation from a teacher's top logits.  For row i with temperature t, over its entries k with an index
 * in [0, vocab):
 *   p_k  = softmax_k(top_logits_ik / t)         the teacher, renormalised over the entries that it has
 *   q_j  = softmax_j(logits_ij / t)             the student, over the whole vocabulary
 *   loss_i     = t^2 * sum_k p_k (log p_k - log q_index(k))
 *   dlogits_ij = g_i * t * (q_j - sum_{k: index(k) = j} p_k)        with g_i the gradient of loss_i
 * Entries whose index is negative or not below vocab are absent, entries of logit -infinity have p_k = 0; a
 * row with no entry of a positive p_k has loss 0 and gradient 0 whatever its logits are.  An index may appear
 * more than once in a row.  A row with g_i = 0 gets zeros whatever its logits are.  Otherwise NaN and
 * infinity propagate per IEEE 754. */
typedef enum { COLLAGE_DTYPE_BF16 = 0, COLLAGE_DTYPE_F32 = 1 } collage_dtype_t;
typedef struct collage_distill {
    collage_matrix_t logits;         /* [rows, vocab] in logits_dtype                                       */
    collage_matrix_t top_index;      /* [rows, k] of int32_t or int64_t (top_index_bytes = 4 or 8)          */
    collage_matrix_t top_logits;     /* [rows, k] of float; k <= COLLAGE_DISTILL_MAX_TOP (ERR_LIMIT)        */
    collage_dtype_t logits_dtype;
    uint32_t top_index_bytes;
    double temperature;              /* > 0 and finite, as is 1 / (temperature ln 2), in float (ERR_ARG)    */
} collage_distill_t;
#define COLLAGE_DISTILL_MAX_TOP 1024

/* loss: DEVICE float[rows].  lse: DEVICE float[rows] or NULL: log sum_j exp(logits_ij / t), for the backward call.  What its
 * rounding to float takes, 2^-24 of its size, comes back twice as the relative error of q there; where that would pass 2^-17 (lse of 128 or
 * more) the backward call takes maximum and sum from the row itself. */
collage_status_t collage_distill_loss(const collage_distill_t* in, float* loss, float* lse, void* stream);
/* grad_loss: DEVICE float[rows], g_i.  dlogits: [rows, vocab] in logits_dtype; may be the array of logits. */
collage_status_t collage_distill_loss_backward(const collage_distill_t* in, const float* lse, const float* grad_loss,
                                               const collage_matrix_t* dlogits, void* stream);
/* Both in one pass over the logits for the objective sum_i row_weight_i * loss_i: loss[i] receives
 * row_weight_i * loss_i (0 where the weight is 0, and the row's logits are then not read), dlogits the gradient with
 * g_i = row_weight_i.  dlogits may be the array of logits. */
collage_status_t collage_distill_loss_and_grad(const collage_distill_t* in, const float* row_weight, float* loss,
                                               const collage_matrix_t* dlogits, void* stream);

/* ------------------------------------------------------------------------------------------------
 * Norms around a block.  A block's output o joins the stream x, normed, gated and scaled, and the stream is normed for the next
 * block; both norms, the gate and either scale are optional:
 *   n = o / sqrt(mean_j o^2 + eps) * post_weight      (o without post_weight)
 *   r = residual_scale * x + block_scale * A(gate) * n     (without the factor A where there is no gate)
 *   y = r / sqrt(mean_j r^2 + eps) * pre_weight
 * in the arithmetic of the section above, whose rules on matrices, overlaps, errors, streams and capture hold here too. */
typedef enum {
    COLLAGE_GATE_NONE = 0,       /* A(g) = g                    */
    COLLAGE_GATE_SIGMOID = 1,    /* A(g) = 1 / (1 + exp(-g))    */
    COLLAGE_GATE_SILU = 2        /* A(g) = g / (1 + exp(-g))    */
} collage_gate_activation_t;
typedef struct collage_block_norm {
    collage_matrix_t block;          /* o: bfloat16 [rows, cols]                                            */
    collage_matrix_t gate;           /* bfloat16: [rows, cols], [1, cols] (one for each channel), or data NULL: none */
    const void* post_weight;         /* DEVICE bfloat16[cols], or NULL: no norm after the block            */
    const void* pre_weight;          /* DEVICE bfloat16[cols], or NULL: no norm before the next one        */
    double eps;                      /* >= 0 and finite                                                      */
    double residual_scale, block_scale;    /* finite in float                                                */
    collage_gate_activation_t activation;
} collage_block_norm_t;

/*   x       : bfloat16 [rows, cols].    r: bfloat16 [rows, cols], the new stream, rounded.  It may be the array of x or of o.
 *   y       : bfloat16 [rows, cols] or NULL, from r as it was before that rounding; may be the array of o.
 *   y8, y8_scale: y in e4m3 with a scale a row as in collage_add_rms_norm, or both NULL.  y and y8 need pre_weight.
 *   rstd_post, rstd_pre: DEVICE float[rows] or NULL: 1 / rms of o and of r for the backward pass, each only with its weight.
 * Rows of large, small or non-finite values: as in collage_add_rms_norm, for both norms. */
collage_status_t collage_block_norm(const collage_block_norm_t* in, const collage_matrix_t* x, const collage_matrix_t* r,
                                    const collage_matrix_t* y, const collage_matrix_t* y8, float* y8_scale, float* rstd_post,
                                    float* rstd_pre, void* stream);

/* Its backward pass; `in` as in the forward call (eps is not used).
 *   dy      : bfloat16 [rows, cols], gradient of y, or NULL: none came that way (pre_weight, r and rstd_pre are then not used).
 *   dr      : bfloat16 [rows, cols], gradient that reached r on its own way, or NULL.  One of dy and dr is given.
 *   r, rstd_post, rstd_pre: of the forward call; rstd_post with post_weight only.  r is the stream as it was stored, so that 2^-8 of each
 *             of its values, a rounding to bfloat16, goes into the gradients that have r in them: into dpre_weight above all, a sum of dy r
 *             rstd_pre, and in less measure into dx, dblock, dpost_weight and dgate by way of dy.
 *   dx, dblock: bfloat16 [rows, cols] or NULL: gradients of x and o.  Either may be the array of dy or of dr.
 *   dgate   : bfloat16, shaped like the gate, or NULL; for a gate of channels the sum over the rows.
 *   dpost_weight, dpre_weight: DEVICE bfloat16[cols] or NULL.  (Sums over no rows are zeros.)
 *   workspace: DEVICE scratch of at least collage_block_norm_workspace_bytes(cols), 16-byte aligned, needed with dpost_weight,
 *             dpre_weight or the gradient of a gate of channels; nothing in it is kept between calls (ERR_WORKSPACE).
 * A gradient of 8-bit outputs passes straight through.
 * collage_block_norm_backward_from_x takes x of the forward call in the place of r (with the same residual_scale and block_scale), where it is
 * still there (r was not stored over it), and forms r anew from x and o: gradients of r as it was before its rounding. */
size_t collage_block_norm_workspace_bytes(uint64_t cols);
collage_status_t collage_block_norm_backward(const collage_block_norm_t* in, const collage_matrix_t* dy, const collage_matrix_t* dr,
                                             const collage_matrix_t* r, const float* rstd_post, const float* rstd_pre,
                                             const collage_matrix_t* dx, const collage_matrix_t* dblock, const collage_matrix_t* dgate,
                                             void* dpost_weight, void* dpre_weight, void* workspace, size_t workspace_bytes,
                                             void* stream);
collage_status_t collage_block_norm_backward_from_x(const collage_block_norm_t* in, const collage_matrix_t* dy, const collage_matrix_t* dr,
                                                    const collage_matrix_t* x, const float* rstd_post, const float* rstd_pre,
                                                    const collage_matrix_t* dx, const collage_matrix_t* dblock,
                                                    const collage_matrix_t* dgate, void* dpost_weight, void* dpre_weight, void* workspace,
                                                    size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------------------------------
 * Losses on the log-probabilities of sampled tokens: what a token had under the model, the clipped policy objective with a
 * KL term, and the preference loss of pairs of answers.  The rules of the sections above hold.
 *   logp_i = z_iy - log sum_j exp(z_ij),   z = logits / temperature, y = target_i
 * A row whose target is negative or not below vocab is a prompt or padding: its logits are not read, its logp is 0 and its gradient zeros.
 * Rows are taken relative to their largest logit: only differences within a row count, at any size of the logits; entries of
 * -infinity have no probability.  NaN and infinity otherwise propagate per IEEE 754. */
typedef struct collage_tokens {
    collage_matrix_t logits;         /* [rows, vocab] in logits_dtype                                       */
    const void* target;              /* DEVICE int32_t[rows] or int64_t[rows] (target_bytes = 4 or 8)       */
    collage_dtype_t logits_dtype;
    uint32_t target_bytes;
    double temperature;              /* > 0 and finite, as is 1 / (temperature ln 2), in float (ERR_ARG)    */
} collage_tokens_t;

/* logp: DEVICE float[rows].  logp_rest: DEVICE float[rows] or NULL: what logp's rounding to float took (up to 2^-24 of it, which a sum over
 * a sequence adds up).  stats: DEVICE float[rows][2], 8-byte aligned, or NULL, for the backward call: the row's largest logit, and the
 * sum of exp((logit - largest) / temperature) over the row; zeros in rows that are not read. */
collage_status_t collage_token_logp(const collage_tokens_t* in, float* logp, float* logp_rest, float* stats, void* stream);
/* grad_logp: DEVICE float[rows].  dlogits_ij = grad_logp_i / temperature * ([j = y] - exp(logp of token j)): [rows, vocab] in
 * logits_dtype; may be the array of logits.  A row of grad_logp 0 gets zeros whatever its logits are. */
collage_status_t collage_token_logp_backward(const collage_tokens_t* in, const float* stats, const float* grad_logp,
                                             const collage_matrix_t* dlogits, void* stream);

/* With ratio_i = exp(logp_i - old_logp_i) and k_i = ref_logp_i - logp_i,
 *   L_i  = -min(ratio_i A_i, min(max(ratio_i, 1 - clip_low), 1 + clip_high) A_i) + kl_weight * kl_i,    kl_i = exp(k_i) - k_i - 1
 *   loss_i = row_weight_i * L_i,   dlogits = the gradient of sum_i loss_i, old_logp, ref_logp and A being constants.
 * Where both terms of the minimum are equal the gradient is that of the first.  A row with A_i = 0 has no policy term.
 * Without old_logp the samples are the model's own: ratio is 1, with the gradient of a ratio.  Without ref_logp there is no KL
 * term (kl_weight has to be 0, kl NULL).  Everything a row's scalars need is taken from logp in 64 bits. */
typedef struct collage_policy {
    const float* old_logp;           /* DEVICE float[rows] or NULL    */
    const float* ref_logp;           /* DEVICE float[rows] or NULL    */
    const float* advantage;          /* A: DEVICE float[rows]         */
    const float* row_weight;         /* DEVICE float[rows]            */
    double clip_low, clip_high;      /* 0 <= clip_low <= 1, clip_high >= 0 (infinity: no bound), in float     */
    double kl_weight;                /* >= 0 and finite, in float     */
} collage_policy_t;
/* One pass over the logits.  loss: DEVICE float[rows].  logp, kl: DEVICE float[rows] or NULL.  dlogits: [rows, vocab] in
 * logits_dtype; may be the array of logits.  A row of weight 0 (or without a target) is not read: loss, logp and kl are 0 there,
 * its gradient zeros. */
collage_status_t collage_policy_loss_and_grad(const collage_tokens_t* in, const collage_policy_t* policy, float* loss, float* logp,
                                              float* kl, const collage_matrix_t* dlogits, void* stream);

/* Pairs of answers: sequence 2p is the preferred and 2p + 1 the other answer of pair p; sequence s has rows [offsets[s], offsets[s+1]).
 *   S_s = sum over its rows that have a target of (logp + logp_rest - ref_logp), divided by their number (at least 1) if average
 *   log_ratio_p = S_2p - S_2p+1,   h = beta * log_ratio_p - margin
 *   loss_p = pair_weight_p * (-(1 - label_smoothing) log sigmoid(h) - label_smoothing log sigmoid(-h))
 *   grad_logp = the gradient of sum_p loss_p; 0 in rows without a target and in rows of no sequence.
 * A pair of weight 0 takes no part: its loss and gradients are 0 whatever its log-probabilities are (log_ratio is what it is).
 * offsets ascend within [0, rows]; others are taken into that range and a sequence that would end before it begins as empty (then
 * the gradients of rows that several sequences or none would own are undefined).  Sums are in 64 bits and in a fixed order. */
typedef struct collage_preference {
    const float* logp;               /* DEVICE float[rows]                                                   */
    const float* logp_rest;          /* DEVICE float[rows] or NULL: zeros                                    */
    const float* ref_logp;           /* DEVICE float[rows] or NULL: zeros                                    */
    const void* target;              /* of collage_tokens_t, with its vocab: which rows count                */
    const void* offsets;             /* DEVICE int32_t or int64_t [2 * pairs + 1] (offset_bytes = 4 or 8)    */
    const float* pair_weight;        /* DEVICE float[pairs] or NULL: ones                                    */
    uint64_t rows, vocab, pairs;     /* rows and vocab below 2^31, pairs below 2^30 (ERR_LIMIT)              */
    uint32_t target_bytes, offset_bytes;
    double beta, margin, label_smoothing;      /* finite in float; 0 <= label_smoothing <= 1                 */
    int average;
} collage_preference_t;
/* loss: DEVICE float[pairs].  log_ratio: DEVICE float[pairs] or NULL.  grad_logp: DEVICE float[rows] or NULL. */
collage_status_t collage_preference_loss(const collage_preference_t* in, float* loss, float* log_ratio, float* grad_logp, void* stream);

/* ------------------------------------------------------------------------------------------------
 * AdamW over many tensors at once, with optimizer states in 8 bits or in 32, and the gradients' norm for clipping.  Ordinary mixed
 * precision next to Algorithm 2, for the storage forms that it does not have; scalars are evaluated in double and cast to float.
 *   g = grad * grad_scale;   m' = beta1 m + (1 - beta1) g;   v' = beta2 v + (1 - beta2) g^2
 *   x' = x - lr (m' / (1 - beta1^t) / (sqrt(v' / (1 - beta2^t)) + eps) + weight_decay x)
 * The parameter, by `rest`: NONE  x = theta, theta' = RN_bf16(x');
 *                           BF16  x = theta + rest, a pair as in option B: theta' = RN_bf16(x'), rest' = RN_bf16(x' - theta'),
 *                                 with x' as the sum of theta, rest, -lr q and the decay.  q is the float quotient of RN(m' k1) and
 *                                 RN(RN(sqrt(v') k2) + eps), or of RN(m' k1) and sqrt(RN(v' k3 + eps)) with EPS_INSIDE_SQRT, where k1, k2 and k3 are
 *                                 1 / (1 - beta1^t), 1 / sqrt(1 - beta2^t) and 1 / (1 - beta2^t) as floats; lr q is not rounded.  The decay,
 *                                 lr weight_decay as a float times theta + rest as a float, is off by 2^-22 of itself at most, the sum by 2^-46:
 *                                 theta' is the nearest value unless x' is that close to half-way;
 *                           F32   x = rest, a master weight: rest' = x', theta' = RN_bf16(x') (theta is not read).
 * The states, by `state`: F32   m and v are floats; with rest NONE or F32 the results are collage_adamw_step_fp32's, bit for bit.
 *                         E4M3  m and v are codes of 8 bits with a float scale for each 256 elements of their tensor (the last
 *                               group of a tensor may be shorter):  m = m_code * m_scale,  sqrt(v) = v_code * v_scale, stored again
 *                               as scale = max / 448 and codes of m' / scale, to nearest even, and of u = sqrt(v') / scale (by way of 1 / 448 and
 *                               448 / max as floats: each is off by a unit or two of its last place), u at least 2^-9
 *                               where v' is not 0, rounded down to a multiple of its spacing s after s * d has been added, 0 <= d < 1
 *                               random (448 at most).  The root moves by less than a code's step in a step of beta2 = 0.999; rounding to nearest would never
 *                               move it.  A group whose largest |m'| (or sqrt(v')) is below 2^-100 is stored as zeros with scale 0.
 *                               A gradient whose square is no finite float makes its group's roots NaN from then on, and the group's
 *                               parameters from the next step at the latest.  (Of F32 it makes v infinite, and the quotient 0 while m is finite.)
 * d has 16 bits, of a fixed function of seed, step and position: with mix(x) on 32 bits x ^= x >> 16, x *= 0x6A09E667,
 * x ^= x >> 15, x *= 0xB504F333, x ^= x >> 16 and key = mix(seed_lo + mix(seed_hi + mix(step_lo + mix(step_hi)))), element P of
 * the plan has the lower (even P) or upper half of mix(lo + mix(hi + key)), where hi and lo are the words of P / 2.  A plan counts its
 * elements tensor by tensor in the order given, each tensor's beginning rounded up to a multiple of 256.  The same call gives the same bits.
 * Of hyper->flags EPS_INSIDE_SQRT is taken, and the kernel-choice flags are ignored; hyper->edq_out has to be NULL (ERR_ARG). */
typedef enum { COLLAGE_STATE_F32 = 0, COLLAGE_STATE_E4M3 = 1 } collage_adam_state_t;
typedef enum { COLLAGE_REST_NONE = 0, COLLAGE_REST_BF16 = 1, COLLAGE_REST_F32 = 2 } collage_adam_rest_t;
typedef struct collage_adam_tensor {
    void* theta;             /* DEVICE bfloat16[n]                                                                   */
    void* rest;              /* DEVICE bfloat16[n] or float[n] by the plan's form; NULL for REST_NONE                 */
    void* m;                 /* DEVICE float[n], or e4m3[n], one byte each                                            */
    void* v;                 /* as m                                                                                 */
    float* m_scale;          /* DEVICE float[(n + 255) / 256] for STATE_E4M3, else NULL                               */
    float* v_scale;
    const void* grad;        /* DEVICE bfloat16[n], read only                                                        */
    uint64_t n;
} collage_adam_tensor_t;
typedef struct collage_adam_plan collage_adam_plan_t;   /* opaque; owns a small device table */

/* As collage_plan_create: copies the HOST array, allocates and synchronises; the plan belongs to the current device.  States begin as zeros
 * (codes, scales and floats alike).
 * Errors: ERR_NULL, ERR_ARG (num < 0, unknown form, arrays that the form does not have, misaligned elements, more than 2^32 - 1
 * chunks of 4096 elements), ERR_ALIAS, ERR_LIMIT (no host memory), ERR_ARCH, ERR_CUDA. */
collage_status_t collage_adam_plan_create(const collage_adam_tensor_t* tensors, int num, collage_adam_state_t state,
                                          collage_adam_rest_t rest, collage_adam_plan_t** out_plan);
collage_status_t collage_adam_plan_destroy(collage_adam_plan_t* plan);

/* One step of all the plan's tensors in one launch.  grad_scale: DEVICE float or NULL (1): what every gradient is taken times, such
 * as the factor of collage_adam_grad_norm.  `seed` matters for STATE_E4M3 only.  Scalars, step and seed are recorded by stream capture.
 * Errors: ERR_NULL, ERR_ARG (step 0, hyper range, another device than the plan's), ERR_ALIAS (grad_scale within an array that is
 * written), ERR_ARCH, ERR_CUDA. */
collage_status_t collage_adam_step(const collage_adam_plan_t* plan, const collage_hyper_t* hyper, uint64_t step, uint64_t seed,
                                   const float* grad_scale, void* stream);

/* norm: DEVICE float: sqrt of the sum of squares of all gradients of the plan.  grad_scale: DEVICE float or NULL: min(1, max_norm /
 * norm), 1 for a norm of 0, NaN for a NaN.  max_norm > 0 (infinity: never clipped).  Squares and sums do not overflow; the order of sums is fixed.
 * `workspace` is one of collage_workspace_bytes(), cleared once by collage_workspace_init, as for the EDQ reduction.
 * Errors: ERR_NULL, ERR_ARG, ERR_ALIAS, ERR_WORKSPACE, ERR_ARCH, ERR_CUDA. */
collage_status_t collage_adam_grad_norm(const collage_adam_plan_t* plan, double max_norm, float* norm, float* grad_scale,
                                        void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* COLLAGE_H_ */

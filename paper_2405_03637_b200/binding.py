"""Thin ctypes binding of the CUDA library: same names as ``include/collage.h``, argument marshalling only.

Tensors are ``torch.bfloat16`` CUDA tensors (or anything with ``data_ptr()``); torch supplies
device memory and streams, every step of the computation runs in the library's kernels.
There is no fallback: if the shared library has not been built, loading raises.
"""
from __future__ import annotations

import ctypes
import math
import struct
from pathlib import Path

_LIB_PATH = Path(__file__).resolve().parent / "libcollage_b200.so"      # the in-tree build

OK, ERR_NULL, ERR_ARG, ERR_ALIAS, ERR_ARCH, ERR_CUDA, ERR_WORKSPACE, ERR_LIMIT = range(8)
BF16, LIGHT, PLUS, KAHAN, PLUS_FP32_REGISTERS = 0, 1, 2, 3, 4
FLAG_EPS_INSIDE_SQRT, FLAG_TWOSUM_GROW, FLAG_DECAY_BY_GROW = 1, 2, 4
FLAG_PIPELINE_KERNEL, FLAG_DIRECT_KERNEL, FLAG_LARGE_TILES = 8, 16, 32
OP_ADD, OP_SUB, OP_MUL, OP_DIV, OP_SQRT, OP_FMA = range(6)
ACT_SILU, ACT_GELU_TANH = 0, 1
DTYPE_BF16, DTYPE_F32 = 0, 1
DISTILL_MAX_TOP = 1024
GATE_NONE, GATE_SIGMOID, GATE_SILU = 0, 1, 2
STATE_F32, STATE_E4M3 = 0, 1
REST_NONE, REST_BF16, REST_F32 = 0, 1, 2
ADAM_GROUP = 256            # elements of a tensor that share a scale of its 8-bit states
SCALAR_NAMES = ("b1", "c1", "b2", "c2", "b2h", "b2l", "bc1", "bc2", "a", "lam", "eps")

EXPORTS = (
    "collage_status_string", "collage_derive_scalars", "collage_workspace_bytes", "collage_adamw_step",
    "collage_adamw_step_host", "collage_adamw_step_fp32",
    "collage_plan_create", "collage_adamw_step_multi", "collage_plan_destroy", "collage_plan_num_elements",
    "collage_plan_num_chunks", "collage_plan_set_replicas", "collage_plan_workspace_bytes", "collage_adamw_step_multi_per_tensor",
    "collage_fast_two_sum", "collage_two_sum", "collage_two_prod", "collage_grow",
    "collage_scaling", "collage_mul", "collage_renormalize", "collage_rounded_op", "collage_edq",
    "collage_selftest", "collage_pipeline_fault", "collage_edq_static", "collage_wait_timeout_selftest",
    "collage_workspace_init", "collage_edq_combine", "collage_build_flavor", "collage_enable_peer_access",
    "collage_add_rms_norm", "collage_add_rms_norm_backward", "collage_rms_norm_workspace_bytes", "collage_quantize_rows",
    "collage_gated_ffn", "collage_gated_ffn_backward", "collage_gated_ffn_e4m3",
    "collage_distill_loss", "collage_distill_loss_backward", "collage_distill_loss_and_grad",
    "collage_block_norm", "collage_block_norm_backward", "collage_block_norm_backward_from_x", "collage_block_norm_workspace_bytes",
    "collage_token_logp", "collage_token_logp_backward", "collage_policy_loss_and_grad", "collage_preference_loss",
    "collage_adam_plan_create", "collage_adam_plan_destroy", "collage_adam_step", "collage_adam_grad_norm",
)


class Hyper(ctypes.Structure):
    """collage_hyper_t"""
    _fields_ = [("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double),
                ("eps", ctypes.c_double), ("weight_decay", ctypes.c_double), ("flags", ctypes.c_uint32),
                ("edq_out", ctypes.c_void_p), ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t)]


class Edq(ctypes.Structure):
    """collage_edq_t"""
    _fields_ = [("dot", ctypes.c_double), ("sumsq", ctypes.c_double), ("edq", ctypes.c_double),
                ("n", ctypes.c_uint64), ("lost", ctypes.c_uint64), ("fault", ctypes.c_uint64)]


EDQ_RECORD_BYTES = ctypes.sizeof(Edq)


class Tensor(ctypes.Structure):
    """collage_tensor_t"""
    _fields_ = [("x_hi", ctypes.c_void_p), ("x_lo", ctypes.c_void_p), ("m", ctypes.c_void_p),
                ("v_hi", ctypes.c_void_p), ("v_lo", ctypes.c_void_p), ("grad", ctypes.c_void_p),
                ("n", ctypes.c_uint64)]


class Matrix(ctypes.Structure):
    """collage_matrix_t"""
    _fields_ = [("data", ctypes.c_void_p), ("rows", ctypes.c_uint64), ("cols", ctypes.c_uint64), ("ld", ctypes.c_uint64)]


class Distill(ctypes.Structure):
    """collage_distill_t"""
    _fields_ = [("logits", Matrix), ("top_index", Matrix), ("top_logits", Matrix), ("logits_dtype", ctypes.c_int),
                ("top_index_bytes", ctypes.c_uint32), ("temperature", ctypes.c_double)]


class BlockNorm(ctypes.Structure):
    """collage_block_norm_t"""
    _fields_ = [("block", Matrix), ("gate", Matrix), ("post_weight", ctypes.c_void_p), ("pre_weight", ctypes.c_void_p),
                ("eps", ctypes.c_double), ("residual_scale", ctypes.c_double), ("block_scale", ctypes.c_double), ("activation", ctypes.c_int)]


class Tokens(ctypes.Structure):
    """collage_tokens_t"""
    _fields_ = [("logits", Matrix), ("target", ctypes.c_void_p), ("logits_dtype", ctypes.c_int), ("target_bytes", ctypes.c_uint32),
                ("temperature", ctypes.c_double)]


class Policy(ctypes.Structure):
    """collage_policy_t"""
    _fields_ = [("old_logp", ctypes.c_void_p), ("ref_logp", ctypes.c_void_p), ("advantage", ctypes.c_void_p), ("row_weight", ctypes.c_void_p),
                ("clip_low", ctypes.c_double), ("clip_high", ctypes.c_double), ("kl_weight", ctypes.c_double)]


class Preference(ctypes.Structure):
    """collage_preference_t"""
    _fields_ = [("logp", ctypes.c_void_p), ("logp_rest", ctypes.c_void_p), ("ref_logp", ctypes.c_void_p), ("target", ctypes.c_void_p), ("offsets", ctypes.c_void_p),
                ("pair_weight", ctypes.c_void_p), ("rows", ctypes.c_uint64), ("vocab", ctypes.c_uint64), ("pairs", ctypes.c_uint64),
                ("target_bytes", ctypes.c_uint32), ("offset_bytes", ctypes.c_uint32), ("beta", ctypes.c_double), ("margin", ctypes.c_double),
                ("label_smoothing", ctypes.c_double), ("average", ctypes.c_int)]


class AdamTensor(ctypes.Structure):
    """collage_adam_tensor_t"""
    _fields_ = [("theta", ctypes.c_void_p), ("rest", ctypes.c_void_p), ("m", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("m_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p), ("grad", ctypes.c_void_p), ("n", ctypes.c_uint64)]


class CollageError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: status {status} ({status_string(status)})")


_lib = None
_packed = None              # the same library; its functions take collage_matrix_t and collage_distill_t as packed bytes
_lib_path = _LIB_PATH


def load(path) -> ctypes.CDLL:
    """Use another build of the same sources (``build.py --out``) instead of the in-tree library.

    Only an explicit call selects it (the benchmark's ``--lib``); nothing in the environment can swap
    the library under a caller.  Must come before the first use of the library in this process.
    """
    global _lib_path
    if _lib is not None:
        raise RuntimeError("the library is already loaded; call load() before any other function")
    _lib_path = Path(path).resolve()
    return lib()


def lib() -> ctypes.CDLL:
    """The loaded CUDA library; raises if it has not been built (there is no other path)."""
    global _lib, _packed
    if _lib is None:
        if not _lib_path.exists():
            raise RuntimeError(f"{_lib_path} is missing: build it with `python -m paper_2405_03637_b200.build` "
                               "(this package has no CPU or PyTorch fallback)")
        L = ctypes.CDLL(str(_lib_path))
        vp, u64, i32 = ctypes.c_void_p, ctypes.c_uint64, ctypes.c_int
        L.collage_status_string.restype = ctypes.c_char_p
        L.collage_status_string.argtypes = [i32]
        L.collage_derive_scalars.argtypes = [ctypes.POINTER(Hyper), u64, ctypes.POINTER(ctypes.c_uint16)]
        L.collage_workspace_bytes.restype = ctypes.c_size_t
        L.collage_workspace_bytes.argtypes = [u64]
        L.collage_adamw_step.argtypes = [vp, vp, vp, vp, vp, vp, u64, ctypes.POINTER(Hyper), u64, i32, vp]
        L.collage_adamw_step_host.argtypes = [vp, vp, vp, vp, vp, vp, u64, ctypes.POINTER(Hyper), u64, i32, vp,
                                              ctypes.c_size_t, vp]
        L.collage_adamw_step_fp32.argtypes = [vp, vp, vp, vp, vp, u64, ctypes.POINTER(Hyper), u64, vp]
        L.collage_plan_create.argtypes = [ctypes.POINTER(Tensor), i32, ctypes.c_uint32, ctypes.POINTER(vp)]
        L.collage_adamw_step_multi.argtypes = [vp, ctypes.POINTER(Hyper), u64, i32, vp]
        L.collage_plan_destroy.argtypes = [vp]
        L.collage_plan_num_elements.restype = u64
        L.collage_plan_num_elements.argtypes = [vp]
        L.collage_plan_num_chunks.restype = u64
        L.collage_plan_num_chunks.argtypes = [vp]
        L.collage_plan_set_replicas.argtypes = [vp, ctypes.POINTER(vp), i32]
        L.collage_plan_workspace_bytes.restype = ctypes.c_size_t
        L.collage_plan_workspace_bytes.argtypes = [vp]
        L.collage_adamw_step_multi_per_tensor.argtypes = [vp, ctypes.POINTER(Hyper), u64, i32, vp, i32, vp,
                                                          ctypes.c_size_t, vp]
        for name in ("collage_fast_two_sum", "collage_two_sum", "collage_two_prod", "collage_renormalize"):
            getattr(L, name).argtypes = [vp, vp, vp, vp, u64, vp]
        L.collage_grow.argtypes = [vp, vp, vp, vp, vp, u64, vp]
        L.collage_scaling.argtypes = [vp, vp, vp, vp, vp, u64, vp]
        L.collage_mul.argtypes = [vp, vp, vp, vp, vp, vp, u64, vp]
        L.collage_rounded_op.argtypes = [i32, vp, vp, vp, vp, u64, vp]
        L.collage_edq.argtypes = [vp, vp, vp, vp, vp, u64, vp, vp, ctypes.c_size_t, vp]
        L.collage_edq_static.argtypes = [vp, vp, vp, vp, vp, u64, vp, vp]
        L.collage_selftest.argtypes = [ctypes.POINTER(ctypes.c_uint64), vp]
        L.collage_pipeline_fault.argtypes = [ctypes.POINTER(ctypes.c_uint32)]
        L.collage_wait_timeout_selftest.argtypes = [ctypes.c_uint32, ctypes.c_void_p]
        L.collage_workspace_init.argtypes = [vp, ctypes.c_size_t, vp]
        L.collage_edq_combine.argtypes = [ctypes.POINTER(Edq), i32, ctypes.POINTER(Edq)]
        L.collage_build_flavor.restype = ctypes.c_char_p
        L.collage_build_flavor.argtypes = []
        L.collage_enable_peer_access.argtypes = [i32]
        L.collage_adam_plan_create.argtypes = [ctypes.POINTER(AdamTensor), i32, i32, i32, ctypes.POINTER(vp)]
        L.collage_adam_plan_destroy.argtypes = [vp]
        _declare_operators(L, *[ctypes.POINTER(s) for s in (Matrix, Distill, BlockNorm, Tokens, Policy, Preference)])
        _packed = ctypes.CDLL(str(_lib_path))
        _declare_operators(_packed, *[ctypes.c_char_p] * 6)
        _lib = L
    return _lib


def _declare_operators(L, mp, dp, bp, tp, pp, rp):
    """Argument types of the training-step operators; `mp`, `dp`, ...: how matrices and the structures of arguments are passed."""
    vp, i32, f64, size = ctypes.c_void_p, ctypes.c_int, ctypes.c_double, ctypes.c_size_t
    L.collage_block_norm.argtypes = [bp, mp, mp, mp, mp, vp, vp, vp, vp]
    L.collage_block_norm_workspace_bytes.restype = size
    L.collage_block_norm_workspace_bytes.argtypes = [ctypes.c_uint64]
    L.collage_block_norm_backward.argtypes = [bp, mp, mp, mp, vp, vp, mp, mp, mp, vp, vp, vp, size, vp]
    L.collage_block_norm_backward_from_x.argtypes = [bp, mp, mp, mp, vp, vp, mp, mp, mp, vp, vp, vp, size, vp]
    L.collage_token_logp.argtypes = [tp, vp, vp, vp, vp]
    L.collage_token_logp_backward.argtypes = [tp, vp, vp, mp, vp]
    L.collage_policy_loss_and_grad.argtypes = [tp, pp, vp, vp, vp, mp, vp]
    L.collage_preference_loss.argtypes = [rp, vp, vp, vp, vp]
    L.collage_adam_step.argtypes = [vp, ctypes.POINTER(Hyper), ctypes.c_uint64, ctypes.c_uint64, vp, vp]
    L.collage_adam_grad_norm.argtypes = [vp, f64, vp, vp, vp, size, vp]
    L.collage_add_rms_norm.argtypes = [mp, mp, vp, ctypes.c_double, mp, mp, mp, vp, vp, vp]
    L.collage_rms_norm_workspace_bytes.restype = ctypes.c_size_t
    L.collage_rms_norm_workspace_bytes.argtypes = [ctypes.c_uint64]
    L.collage_add_rms_norm_backward.argtypes = [mp, mp, vp, vp, mp, mp, vp, vp, ctypes.c_size_t, vp]
    L.collage_quantize_rows.argtypes = [mp, mp, vp, vp]
    L.collage_gated_ffn.argtypes = [mp, mp, mp, mp, mp, mp, i32, vp]
    L.collage_gated_ffn_backward.argtypes = [mp] * 11 + [i32, vp]
    L.collage_gated_ffn_e4m3.argtypes = [mp, vp, mp, vp, mp, vp, mp, i32, vp]
    L.collage_distill_loss.argtypes = [dp, vp, vp, vp]
    L.collage_distill_loss_backward.argtypes = [dp, vp, vp, mp, vp]
    L.collage_distill_loss_and_grad.argtypes = [dp, vp, vp, mp, vp]


def _ptr(t):
    if t is None:
        return None
    if isinstance(t, int):
        return t
    if hasattr(t, "cuda_stream"):      # torch.cuda.Stream
        return t.cuda_stream
    return t.data_ptr()


def _check(status: int, where: str):
    if status != OK:
        raise CollageError(status, where)


def status_string(status: int) -> str:
    return lib().collage_status_string(int(status)).decode()


def make_hyper(lr, beta1, beta2, eps, weight_decay, flags=0, edq_out=None, workspace=None) -> Hyper:
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    return Hyper(lr, beta1, beta2, eps, weight_decay, flags, _ptr(edq_out), _ptr(workspace), ws_bytes)


def derive_scalars(hyper: Hyper, step: int) -> dict:
    out = (ctypes.c_uint16 * 11)()
    _check(lib().collage_derive_scalars(ctypes.byref(hyper), step, out), "collage_derive_scalars")
    return dict(zip(SCALAR_NAMES, (int(v) for v in out)))


def workspace_bytes(n_total: int = 0) -> int:
    return int(lib().collage_workspace_bytes(n_total))


def workspace_init(workspace, stream=None):
    """Clear an EDQ workspace (a CUDA uint8 tensor): needed once, before its first use."""
    _check(lib().collage_workspace_init(_ptr(workspace), workspace.numel() * workspace.element_size(), _ptr(stream)),
           "collage_workspace_init")


def _record(rec: Edq) -> dict:
    return dict(dot=rec.dot, sumsq=rec.sumsq, edq=rec.edq, n=int(rec.n), lost=int(rec.lost), fault=int(rec.fault))


def edq_combine(parts) -> dict:
    """EDQ record of the union of disjoint parameter sets from their records (dicts with dot, sumsq, n, lost)."""
    arr = (Edq * max(len(parts), 1))()
    for i, p in enumerate(parts):
        arr[i] = Edq(p["dot"], p["sumsq"], p.get("edq", 0.0), p.get("n", 0), p["lost"], p.get("fault", 0))
    out = Edq()
    _check(lib().collage_edq_combine(arr, len(parts), ctypes.byref(out)), "collage_edq_combine")
    return _record(out)


def build_flavor() -> str:
    return lib().collage_build_flavor().decode()


def adamw_step(x_hi, x_lo, m, v_hi, v_lo, grad, n, hyper: Hyper, step: int, strategy: int, stream=None):
    _check(lib().collage_adamw_step(_ptr(x_hi), _ptr(x_lo), _ptr(m), _ptr(v_hi), _ptr(v_lo), _ptr(grad), n,
                                    ctypes.byref(hyper), step, strategy, _ptr(stream)), "collage_adamw_step")


def adamw_step_host(x_hi, x_lo, m, v_hi, v_lo, grad, n, hyper: Hyper, step: int, strategy: int, staging, stream=None):
    """Host-resident state (pinned CPU tensors); `staging` is a CUDA uint8 tensor; hyper.edq_out is a host address."""
    _check(lib().collage_adamw_step_host(_ptr(x_hi), _ptr(x_lo), _ptr(m), _ptr(v_hi), _ptr(v_lo), _ptr(grad), n,
                                         ctypes.byref(hyper), step, strategy, _ptr(staging),
                                         staging.numel() * staging.element_size(), _ptr(stream)),
           "collage_adamw_step_host")


def adamw_step_fp32(theta, master, m, v, grad, n, hyper: Hyper, step: int, stream=None):
    """Comparator option D (master: float32 CUDA tensor) / D^-MW (master None); m, v float32, theta, grad bfloat16."""
    _check(lib().collage_adamw_step_fp32(_ptr(theta), _ptr(master), _ptr(m), _ptr(v), _ptr(grad), n, ctypes.byref(hyper),
                                         step, _ptr(stream)), "collage_adamw_step_fp32")


def plan_create(tensors, chunk_elems: int = 0) -> int:
    """tensors: list of (x_hi, x_lo, m, v_hi, v_lo, grad, n); returns the opaque plan handle."""
    arr = (Tensor * max(len(tensors), 1))()
    for i, (x_hi, x_lo, m, v_hi, v_lo, grad, n) in enumerate(tensors):
        arr[i] = Tensor(_ptr(x_hi), _ptr(x_lo), _ptr(m), _ptr(v_hi), _ptr(v_lo), _ptr(grad), n)
    plan = ctypes.c_void_p()
    _check(lib().collage_plan_create(arr, len(tensors), chunk_elems, ctypes.byref(plan)), "collage_plan_create")
    return plan.value


def adamw_step_multi(plan: int, hyper: Hyper, step: int, strategy: int, stream=None):
    _check(lib().collage_adamw_step_multi(plan, ctypes.byref(hyper), step, strategy, _ptr(stream)),
           "collage_adamw_step_multi")


def plan_set_replicas(plan: int, replicas):
    """replicas: list (one per replica) of lists (one per tensor of the plan, None for empty tensors) of tensors/addresses."""
    flat = [(_ptr(t) or 0) for rep in replicas for t in rep]
    arr = (ctypes.c_void_p * max(len(flat), 1))(*flat)
    _check(lib().collage_plan_set_replicas(plan, arr, len(replicas)), "collage_plan_set_replicas")


def enable_peer_access(peer_device: int):
    """Let kernels of the current device store into `peer_device`'s memory (set-up for replicas on other GPUs)."""
    _check(lib().collage_enable_peer_access(peer_device), "collage_enable_peer_access")


def plan_workspace_bytes(plan: int) -> int:
    return int(lib().collage_plan_workspace_bytes(plan))


def adamw_step_multi_per_tensor(plan: int, hyper: Hyper, step: int, strategy: int, per_tensor_out, num: int,
                                chunk_workspace, stream=None):
    """per_tensor_out: CUDA uint8 tensor of num * EDQ_RECORD_BYTES bytes; chunk_workspace: CUDA uint8 tensor."""
    _check(lib().collage_adamw_step_multi_per_tensor(plan, ctypes.byref(hyper), step, strategy, _ptr(per_tensor_out), num,
                                                     _ptr(chunk_workspace),
                                                     chunk_workspace.numel() * chunk_workspace.element_size(),
                                                     _ptr(stream)), "collage_adamw_step_multi_per_tensor")


def read_edq_array(dev_bytes, num: int) -> list:
    """Decode num consecutive device collage_edq_t records."""
    raw = dev_bytes.detach().cpu().numpy().tobytes()
    out = []
    for i in range(num):
        out.append(_record(Edq.from_buffer_copy(raw[i * ctypes.sizeof(Edq):(i + 1) * ctypes.sizeof(Edq)])))
    return out


def plan_destroy(plan: int):
    _check(lib().collage_plan_destroy(plan), "collage_plan_destroy")


def plan_num_elements(plan: int) -> int:
    return int(lib().collage_plan_num_elements(plan))


def plan_num_chunks(plan: int) -> int:
    return int(lib().collage_plan_num_chunks(plan))


def fast_two_sum(a, b, hi, lo, n, stream=None):
    _check(lib().collage_fast_two_sum(_ptr(a), _ptr(b), _ptr(hi), _ptr(lo), n, _ptr(stream)), "collage_fast_two_sum")


def two_sum(a, b, hi, lo, n, stream=None):
    _check(lib().collage_two_sum(_ptr(a), _ptr(b), _ptr(hi), _ptr(lo), n, _ptr(stream)), "collage_two_sum")


def two_prod(a, b, hi, lo, n, stream=None):
    _check(lib().collage_two_prod(_ptr(a), _ptr(b), _ptr(hi), _ptr(lo), n, _ptr(stream)), "collage_two_prod")


def renormalize(hi_in, lo_in, hi, lo, n, stream=None):
    _check(lib().collage_renormalize(_ptr(hi_in), _ptr(lo_in), _ptr(hi), _ptr(lo), n, _ptr(stream)),
           "collage_renormalize")


def grow(x, y, a, u, v, n, stream=None):
    _check(lib().collage_grow(_ptr(x), _ptr(y), _ptr(a), _ptr(u), _ptr(v), n, _ptr(stream)), "collage_grow")


def scaling(v, a1, a2, x, e, n, stream=None):
    _check(lib().collage_scaling(_ptr(v), _ptr(a1), _ptr(a2), _ptr(x), _ptr(e), n, _ptr(stream)), "collage_scaling")


def mul(a1, a2, b1, b2, x, e, n, stream=None):
    _check(lib().collage_mul(_ptr(a1), _ptr(a2), _ptr(b1), _ptr(b2), _ptr(x), _ptr(e), n, _ptr(stream)), "collage_mul")


def rounded_op(op, a, b, c, out, n, stream=None):
    _check(lib().collage_rounded_op(op, _ptr(a), _ptr(b), _ptr(c), _ptr(out), n, _ptr(stream)), "collage_rounded_op")


def edq(old_hi, old_lo, new_hi, new_lo, delta, n, out_dev, workspace, stream=None):
    ws_bytes = workspace.numel() * workspace.element_size()
    _check(lib().collage_edq(_ptr(old_hi), _ptr(old_lo), _ptr(new_hi), _ptr(new_lo), _ptr(delta), n, _ptr(out_dev),
                             _ptr(workspace), ws_bytes, _ptr(stream)), "collage_edq")


def edq_static(old_hi, old_lo, new_hi, new_lo, delta, n, out_dev, stream=None):
    """EDQ with the library's built-in scratch: for callers that cannot allocate a workspace (n <= 2^32)."""
    _check(lib().collage_edq_static(_ptr(old_hi), _ptr(old_lo), _ptr(new_hi), _ptr(new_lo), _ptr(delta), n,
                                    _ptr(out_dev), _ptr(stream)), "collage_edq_static")


def selftest(stream=None) -> dict:
    out = (ctypes.c_uint64 * 6)()
    _check(lib().collage_selftest(out, _ptr(stream)), "collage_selftest")
    return dict(zip(("add", "sub", "mul", "div", "sqrt", "scalar_div"), (int(v) for v in out)))


def pipeline_fault() -> int:
    out = ctypes.c_uint32(0)
    _check(lib().collage_pipeline_fault(ctypes.byref(out)), "collage_pipeline_fault")
    return int(out.value)


def wait_timeout_selftest(limit_ms: int, stream=None):
    _check(lib().collage_wait_timeout_selftest(limit_ms, _ptr(stream)), "collage_wait_timeout_selftest")


def read_edq(edq_dev) -> dict:
    """Copy a device collage_edq_t (a >= EDQ_RECORD_BYTES torch.uint8 CUDA tensor) to the host and decode it."""
    raw = edq_dev.detach().cpu().numpy().tobytes()
    return _record(Edq.from_buffer_copy(raw[:ctypes.sizeof(Edq)]))


# ------------------------------------------------------------------------------------------------------------------------
# Operators of the forward and backward pass.  Matrices are CUDA tensors of two or more dimensions whose last one is
# contiguous; leading dimensions are flattened into rows (a view, never a copy).  What a tensor cannot be described as, or
# is not on the current device or of the type that the operator reads, raises CollageError(ERR_ARG) here; all other checks are
# the library's.  As everywhere in this module, stream=None is the device's default stream; torch's streams do not wait for that
# one, so where another is current (torch.cuda.stream, a graph's capture) the operators want their stream named (ERR_ARG).
# They read and write through addresses: autograd records nothing of them (the backward functions are called by hand or from a
# torch.autograd.Function), and tensors written in the place of others, such as dgate over gate, change without its knowledge.

def _refuse(where: str):
    raise CollageError(ERR_ARG, where)


_BF16 = _F32 = _E4M3 = _I32 = _I64 = None           # torch's types, from the first operator on: the rest of this module does without torch
_current_device = _current_stream = None


def _operators():
    """The library as the operators call it and the current device's number.  First of all in each of them."""
    global _BF16, _F32, _E4M3, _I32, _I64, _current_device, _current_stream
    if _BF16 is None:
        import torch
        lib()
        # (the plain numbers, without checks or objects around them, where torch gives them: 0.1 us in place of 1)
        _current_device, _current_stream = lambda: None, lambda dev: 0
        if torch.cuda.is_available():
            torch.cuda.init()
            _current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
            _current_stream = getattr(torch._C, "_cuda_getCurrentRawStream", lambda dev: torch.cuda.current_stream(dev).cuda_stream)
        _F32, _E4M3, _I32, _I64 = torch.float32, torch.float8_e4m3fn, torch.int32, torch.int64
        _BF16 = torch.bfloat16
    return _packed, _current_device()


_pack_matrix = struct.Struct("QQQQ").pack          # collage_matrix_t: a third of the time that a ctypes structure takes
_pack_distill = struct.Struct("iId").pack
_pack_block_norm = struct.Struct("QQdddi4x").pack      # what follows the matrices in collage_block_norm_t
_pack_tokens = struct.Struct("QiId").pack              # and in collage_tokens_t
_pack_policy = struct.Struct("QQQQddd").pack
_pack_preference = struct.Struct("QQQQQQQQQIIdddi4x").pack
_NO_MATRIX = _pack_matrix(0, 0, 0, 0)


def _flat(t):
    """Leading dimensions as rows (RuntimeError where a view cannot be had)."""
    *lead, cols = t.shape
    return t.view(-1, cols) if cols else t.view(math.prod(lead), 0)


def _matrix(t, dtype, dev, where: str, required: bool = False):
    """collage_matrix_t of a tensor, packed, or None for None."""
    if t is None:
        if required:
            raise CollageError(ERR_NULL, where)
        return None
    if t.dtype is not dtype or t.get_device() != dev:
        _refuse(where)
    shape = t.shape
    if len(shape) != 2:
        if len(shape) < 2:
            _refuse(where)
        try:
            t = _flat(t)
        except RuntimeError:
            _refuse(where)
        shape = t.shape
    rows, cols = shape
    ld, inner = t.stride()
    if inner != 1 or ld < cols or rows <= 1:
        if rows <= 1:
            ld = cols                          # the stride of a single row means nothing, nor that within a single column
        if (inner != 1 and cols > 1) or ld < cols:
            _refuse(where)
    return _pack_matrix(t.data_ptr(), rows, cols, ld)


def _extents(t):
    """Rows and columns of a tensor that _matrix has taken."""
    shape = t.shape
    return shape if len(shape) == 2 else _flat(t).shape


def _vector(t, dtype, length: int, dev, where: str):
    """Address of a contiguous vector of that many elements, or None for None."""
    if t is None:
        return None
    if t.dtype is not dtype or t.get_device() != dev or t.numel() != length or not t.is_contiguous():
        _refuse(where)
    return t.data_ptr()


def _stream(stream, dev, where: str):
    """Address of a stream of the current device, or None for the default stream where that is torch's current one."""
    if stream is None:
        if _current_stream(dev):
            _refuse(f"{where}: stream=None while torch's current stream is not the default one")
        return None
    if getattr(stream, "device_index", dev) != dev:
        _refuse(f"{where}: a stream of another device")
    return _ptr(stream)


def add_rms_norm(x, residual, weight, eps: float, residual_out=None, y=None, y8=None, y8_scale=None, rstd=None, stream=None):
    """r = x + residual; y = r / sqrt(mean(r^2) + eps) * weight in bfloat16 (y) and / or in 8 bits (y8, y8_scale)."""
    w, (L, dev) = "collage_add_rms_norm", _operators()
    mx = _matrix(x, _BF16, dev, w, True)
    rows, cols = _extents(x)
    _check(L.collage_add_rms_norm(mx, _matrix(residual, _BF16, dev, w), _vector(weight, _BF16, cols, dev, w), eps,
                                  _matrix(residual_out, _BF16, dev, w), _matrix(y, _BF16, dev, w), _matrix(y8, _E4M3, dev, w),
                                  _vector(y8_scale, _F32, rows, dev, w), _vector(rstd, _F32, rows, dev, w), _stream(stream, dev, w)), w)


def rms_norm_workspace_bytes(cols: int) -> int:
    return int(lib().collage_rms_norm_workspace_bytes(cols))


def add_rms_norm_backward(dy, r, rstd, weight, dx, dweight, workspace, dresidual=None, stream=None):
    """Gradients of add_rms_norm: r is its residual_out (or x without a residual); dx or dweight may be None."""
    w, (L, dev) = "collage_add_rms_norm_backward", _operators()
    mdy = _matrix(dy, _BF16, dev, w, True)
    ws_bytes = 0
    if workspace is not None:
        ws_bytes = workspace.numel() * workspace.element_size()
        if workspace.get_device() != dev or not workspace.is_contiguous():
            _refuse(w)
    rows, cols = _extents(dy)
    _check(L.collage_add_rms_norm_backward(mdy, _matrix(r, _BF16, dev, w), _vector(rstd, _F32, rows, dev, w),
                                           _vector(weight, _BF16, cols, dev, w), _matrix(dresidual, _BF16, dev, w),
                                           _matrix(dx, _BF16, dev, w), _vector(dweight, _BF16, cols, dev, w), _ptr(workspace),
                                           ws_bytes, _stream(stream, dev, w)), w)


def quantize_rows(x, q, scale, stream=None):
    """q, scale: x in 8 bits (torch.float8_e4m3fn) with one float scale a row."""
    w, (L, dev) = "collage_quantize_rows", _operators()
    mx = _matrix(x, _BF16, dev, w, True)
    _check(L.collage_quantize_rows(mx, _matrix(q, _E4M3, dev, w), _vector(scale, _F32, _extents(x)[0], dev, w), _stream(stream, dev, w)), w)


def gated_ffn(x, w_gate, w_up, h, gate=None, up=None, activation: int = ACT_SILU, stream=None):
    """h = act(x w_gate^T) * (x w_up^T); gate and up, if given, keep the two products for the backward pass."""
    w, (L, dev) = "collage_gated_ffn", _operators()
    _check(L.collage_gated_ffn(_matrix(x, _BF16, dev, w), _matrix(w_gate, _BF16, dev, w), _matrix(w_up, _BF16, dev, w), _matrix(h, _BF16, dev, w),
                               _matrix(gate, _BF16, dev, w), _matrix(up, _BF16, dev, w), activation, _stream(stream, dev, w)), w)


def gated_ffn_backward(dh, x, w_gate, w_up, gate, up, dgate, dup, dx=None, dw_gate=None, dw_up=None, activation: int = ACT_SILU,
                       stream=None):
    """Gradients of gated_ffn; dgate and dup receive the gradients of the two products (they may be gate and up themselves)."""
    w, (L, dev) = "collage_gated_ffn_backward", _operators()
    m = [_matrix(t, _BF16, dev, w) for t in (dh, x, w_gate, w_up, gate, up, dgate, dup, dx, dw_gate, dw_up)]
    _check(L.collage_gated_ffn_backward(*m, activation, _stream(stream, dev, w)), w)


def gated_ffn_e4m3(x8, x_scale, w_gate8, w_gate_scale, w_up8, w_up_scale, h, activation: int = ACT_SILU, stream=None):
    """gated_ffn on 8-bit operands with a scale for each token and each channel, as quantize_rows writes them."""
    w, (L, dev) = "collage_gated_ffn_e4m3", _operators()
    mx, mg, mu = _matrix(x8, _E4M3, dev, w, True), _matrix(w_gate8, _E4M3, dev, w, True), _matrix(w_up8, _E4M3, dev, w, True)
    _check(L.collage_gated_ffn_e4m3(mx, _vector(x_scale, _F32, _extents(x8)[0], dev, w), mg,
                                    _vector(w_gate_scale, _F32, _extents(w_gate8)[0], dev, w), mu,
                                    _vector(w_up_scale, _F32, _extents(w_up8)[0], dev, w), _matrix(h, _BF16, dev, w), activation,
                                    _stream(stream, dev, w)), w)


def _distill(logits, top_index, top_logits, temperature, dev, where):
    """collage_distill_t, packed, and the number of rows."""
    if logits is None or top_index is None or top_logits is None:
        raise CollageError(ERR_NULL, where)
    dtype, index = logits.dtype, top_index.dtype
    if dtype not in (_BF16, _F32) or index not in (_I32, _I64):
        _refuse(where)
    packed = (_matrix(logits, dtype, dev, where) + _matrix(top_index, index, dev, where) + _matrix(top_logits, _F32, dev, where) +
              _pack_distill(DTYPE_BF16 if dtype is _BF16 else DTYPE_F32, 4 if index is _I32 else 8, temperature))
    return packed, _extents(logits)[0]


def distill_loss(logits, top_index, top_logits, temperature: float, loss, lse=None, stream=None):
    """loss[i] = temperature^2 KL(teacher's renormalised top entries || softmax(logits / temperature)) for each row."""
    w, (L, dev) = "collage_distill_loss", _operators()
    d, n = _distill(logits, top_index, top_logits, temperature, dev, w)
    _check(L.collage_distill_loss(d, _vector(loss, _F32, n, dev, w), _vector(lse, _F32, n, dev, w), _stream(stream, dev, w)), w)


def distill_loss_backward(logits, top_index, top_logits, temperature: float, lse, grad_loss, dlogits, stream=None):
    """dlogits from grad_loss (one value a row) and the lse of distill_loss; dlogits may be the logits' own array."""
    w, (L, dev) = "collage_distill_loss_backward", _operators()
    d, n = _distill(logits, top_index, top_logits, temperature, dev, w)
    _check(L.collage_distill_loss_backward(d, _vector(lse, _F32, n, dev, w), _vector(grad_loss, _F32, n, dev, w),
                                           _matrix(dlogits, logits.dtype, dev, w), _stream(stream, dev, w)), w)


def distill_loss_and_grad(logits, top_index, top_logits, temperature: float, row_weight, loss, dlogits, stream=None):
    """loss[i] = row_weight[i] * the row's loss, and dlogits, in one pass; dlogits may be the logits' own array."""
    w, (L, dev) = "collage_distill_loss_and_grad", _operators()
    d, n = _distill(logits, top_index, top_logits, temperature, dev, w)
    _check(L.collage_distill_loss_and_grad(d, _vector(row_weight, _F32, n, dev, w), _vector(loss, _F32, n, dev, w),
                                           _matrix(dlogits, logits.dtype, dev, w), _stream(stream, dev, w)), w)


def _scratch(workspace, dev, where: str):
    """Address and bytes of a workspace of the current device, or None and 0."""
    if workspace is None:
        return None, 0
    if workspace.get_device() != dev or not workspace.is_contiguous():
        _refuse(where)
    return workspace.data_ptr(), workspace.numel() * workspace.element_size()


def _block_norm(block, gate, post_weight, pre_weight, eps, residual_scale, block_scale, activation, dev, where):
    """collage_block_norm_t, packed, and the block's rows and columns."""
    mb, mg = _matrix(block, _BF16, dev, where, True), _matrix(gate, _BF16, dev, where)
    rows, cols = _extents(block)
    return (mb + (mg or _NO_MATRIX) + _pack_block_norm(_vector(post_weight, _BF16, cols, dev, where) or 0, _vector(pre_weight, _BF16, cols, dev, where) or 0,
                                                       eps, residual_scale, block_scale, activation)), rows, cols


def block_norm(x, block, r, gate=None, post_weight=None, pre_weight=None, y=None, y8=None, y8_scale=None, rstd_post=None, rstd_pre=None,
               eps: float = 1e-6, residual_scale: float = 1.0, block_scale: float = 1.0, activation: int = GATE_NONE, stream=None):
    """r = residual_scale x + block_scale A(gate) norm(block) post_weight; y = norm(r) pre_weight in bfloat16 (y) and / or 8 bits (y8, y8_scale).

    gate: one row for all, or a row for each; without post_weight the block's output is not normed, without pre_weight there is no y.
    """
    w, (L, dev) = "collage_block_norm", _operators()
    s, rows, _ = _block_norm(block, gate, post_weight, pre_weight, eps, residual_scale, block_scale, activation, dev, w)
    _check(L.collage_block_norm(s, _matrix(x, _BF16, dev, w, True), _matrix(r, _BF16, dev, w, True), _matrix(y, _BF16, dev, w), _matrix(y8, _E4M3, dev, w),
                                _vector(y8_scale, _F32, rows, dev, w), _vector(rstd_post, _F32, rows, dev, w), _vector(rstd_pre, _F32, rows, dev, w),
                                _stream(stream, dev, w)), w)


def block_norm_workspace_bytes(cols: int) -> int:
    return int(lib().collage_block_norm_workspace_bytes(cols))


def block_norm_backward(dy, r, block, rstd_post, rstd_pre, dx, dblock, dr=None, gate=None, post_weight=None, pre_weight=None, dgate=None,
                        dpost_weight=None, dpre_weight=None, workspace=None, residual_scale: float = 1.0, block_scale: float = 1.0,
                        activation: int = GATE_NONE, stream=None, x=None):
    """Gradients of block_norm from that of y (dy) and that which reached r on its own way (dr); outputs that are None are not computed.

    With r as the forward call stored it, the gradients take in its rounding.  Where x is still there, r=None and x in its place leave that out:
    r is formed anew from x and block.
    """
    w, (L, dev) = "collage_block_norm_backward", _operators()
    if x is not None and r is not None:
        _refuse(f"{w}: r and x")
    s, rows, cols = _block_norm(block, gate, post_weight, pre_weight, 0.0, residual_scale, block_scale, activation, dev, w)
    ws, ws_bytes = _scratch(workspace, dev, w)
    f, stored = (L.collage_block_norm_backward, r) if x is None else (L.collage_block_norm_backward_from_x, x)
    _check(f(s, _matrix(dy, _BF16, dev, w), _matrix(dr, _BF16, dev, w), _matrix(stored, _BF16, dev, w), _vector(rstd_post, _F32, rows, dev, w),
             _vector(rstd_pre, _F32, rows, dev, w), _matrix(dx, _BF16, dev, w), _matrix(dblock, _BF16, dev, w), _matrix(dgate, _BF16, dev, w),
             _vector(dpost_weight, _BF16, cols, dev, w), _vector(dpre_weight, _BF16, cols, dev, w), ws, ws_bytes, _stream(stream, dev, w)), w)


def _index(t, length, dev, where):
    """Address of a contiguous vector of int32 or int64, and the bytes of its elements."""
    if t is None:
        raise CollageError(ERR_NULL, where)
    dtype = t.dtype
    if dtype is not _I32 and dtype is not _I64:
        _refuse(where)
    return _vector(t, dtype, length, dev, where), 4 if dtype is _I32 else 8


def _tokens(logits, target, temperature, dev, where):
    """collage_tokens_t, packed, and the number of rows."""
    if logits is None:
        raise CollageError(ERR_NULL, where)
    dtype = logits.dtype
    if dtype is not _BF16 and dtype is not _F32:
        _refuse(where)
    m = _matrix(logits, dtype, dev, where)
    rows = _extents(logits)[0]
    at, size = _index(target, rows, dev, where)
    return m + _pack_tokens(at, DTYPE_BF16 if dtype is _BF16 else DTYPE_F32, size, temperature), rows


def token_logp(logits, target, temperature: float, logp, stats=None, logp_rest=None, stream=None):
    """logp[i] = log softmax(logits[i] / temperature)[target[i]], 0 where target[i] is no token; stats [rows, 2] for the backward call;
    logp_rest: what logp's rounding to float took, for preference_loss."""
    w, (L, dev) = "collage_token_logp", _operators()
    t, n = _tokens(logits, target, temperature, dev, w)
    _check(L.collage_token_logp(t, _vector(logp, _F32, n, dev, w), _vector(logp_rest, _F32, n, dev, w), _vector(stats, _F32, 2 * n, dev, w), _stream(stream, dev, w)), w)


def token_logp_backward(logits, target, temperature: float, stats, grad_logp, dlogits, stream=None):
    """dlogits from grad_logp (one value a row) and the stats of token_logp; dlogits may be the logits' own array."""
    w, (L, dev) = "collage_token_logp_backward", _operators()
    t, n = _tokens(logits, target, temperature, dev, w)
    _check(L.collage_token_logp_backward(t, _vector(stats, _F32, 2 * n, dev, w), _vector(grad_logp, _F32, n, dev, w),
                                         _matrix(dlogits, logits.dtype, dev, w), _stream(stream, dev, w)), w)


def policy_loss_and_grad(logits, target, temperature: float, advantage, row_weight, loss, dlogits, old_logp=None, ref_logp=None,
                         clip_low: float = 0.2, clip_high: float = 0.2, kl_weight: float = 0.0, logp=None, kl=None, stream=None):
    """loss[i] = row_weight[i] * (clipped policy loss + kl_weight * kl[i]) of each token, and dlogits, in one pass; dlogits may be the logits' own array."""
    w, (L, dev) = "collage_policy_loss_and_grad", _operators()
    t, n = _tokens(logits, target, temperature, dev, w)
    p = _pack_policy(_vector(old_logp, _F32, n, dev, w) or 0, _vector(ref_logp, _F32, n, dev, w) or 0, _vector(advantage, _F32, n, dev, w) or 0,
                     _vector(row_weight, _F32, n, dev, w) or 0, clip_low, clip_high, kl_weight)
    _check(L.collage_policy_loss_and_grad(t, p, _vector(loss, _F32, n, dev, w), _vector(logp, _F32, n, dev, w), _vector(kl, _F32, n, dev, w),
                                          _matrix(dlogits, logits.dtype, dev, w), _stream(stream, dev, w)), w)


def preference_loss(logp, target, vocab: int, offsets, beta: float, loss, grad_logp=None, ref_logp=None, pair_weight=None, margin: float = 0.0,
                    label_smoothing: float = 0.0, average: bool = False, log_ratio=None, logp_rest=None, stream=None):
    """loss[p] = -log sigmoid(beta (S_2p - S_2p+1) - margin) of pairs of sequences [offsets[s], offsets[s + 1]) of rows, S summing logp + logp_rest - ref_logp;
    and grad_logp."""
    w, (L, dev) = "collage_preference_loss", _operators()
    if logp is None or offsets is None:
        raise CollageError(ERR_NULL, w)
    rows, edges = logp.numel(), offsets.numel()
    if edges % 2 == 0 or not 0 <= vocab < 1 << 64:
        _refuse(w)
    pairs = edges // 2
    at, size = _index(target, rows, dev, w)
    edge, edge_size = _index(offsets, edges, dev, w)
    p = _pack_preference(_vector(logp, _F32, rows, dev, w), _vector(logp_rest, _F32, rows, dev, w) or 0, _vector(ref_logp, _F32, rows, dev, w) or 0, at, edge,
                         _vector(pair_weight, _F32, pairs, dev, w) or 0, rows, vocab, pairs, size, edge_size, beta, margin, label_smoothing, bool(average))
    _check(L.collage_preference_loss(p, _vector(loss, _F32, pairs, dev, w), _vector(log_ratio, _F32, pairs, dev, w), _vector(grad_logp, _F32, rows, dev, w),
                                     _stream(stream, dev, w)), w)


# ------------------------------------------------------------------------------------------------------------------------
# AdamW over many tensors with states in 8 or 32 bits.  As plan_create's, a plan's tensors have to outlive it.

def adam_plan_create(tensors) -> int:
    """tensors: list of (theta, rest, m, v, m_scale, v_scale, grad), contiguous CUDA tensors of the current device; returns the plan's handle.

    theta, grad: bfloat16.  rest: None, bfloat16 (a pair's second part) or float32 (master weights), alike for all.  m, v: float32 with
    m_scale and v_scale None, or torch.float8_e4m3fn with a float32 scale for each ADAM_GROUP elements, alike for all; zeros to begin with.
    """
    w, (_, dev) = "collage_adam_plan_create", _operators()
    arr = (AdamTensor * max(len(tensors), 1))()
    state = rest_kind = None
    for i, (theta, rest, m, v, m_scale, v_scale, grad) in enumerate(tensors):
        if theta is None or m is None or v is None or grad is None:
            raise CollageError(ERR_NULL, w)
        kinds = (STATE_F32 if m.dtype is _F32 else STATE_E4M3, REST_NONE if rest is None else REST_BF16 if rest.dtype is _BF16 else REST_F32)
        if i and kinds != (state, rest_kind):
            _refuse(f"{w}: tensors of different forms")
        state, rest_kind = kinds
        n = theta.numel()
        groups = -(-n // ADAM_GROUP)
        code = _F32 if state == STATE_F32 else _E4M3
        arr[i] = AdamTensor(_vector(theta, _BF16, n, dev, w), _vector(rest, _BF16 if rest_kind == REST_BF16 else _F32, n, dev, w), _vector(m, code, n, dev, w),
                            _vector(v, code, n, dev, w), _vector(m_scale, _F32, groups, dev, w), _vector(v_scale, _F32, groups, dev, w),
                            _vector(grad, _BF16, n, dev, w), n)
    plan = ctypes.c_void_p()
    _check(lib().collage_adam_plan_create(arr, len(tensors), state or 0, rest_kind or 0, ctypes.byref(plan)), w)
    return plan.value


def adam_plan_destroy(plan: int):
    _check(lib().collage_adam_plan_destroy(plan), "collage_adam_plan_destroy")


def adam_step(plan: int, hyper: Hyper, step: int, seed: int = 0, grad_scale=None, stream=None):
    """One step of all the plan's tensors; grad_scale: a float32 CUDA tensor of one element that the gradients are taken times."""
    w, (L, dev) = "collage_adam_step", _operators()
    _check(L.collage_adam_step(plan, ctypes.byref(hyper), step, seed, _vector(grad_scale, _F32, 1, dev, w), _stream(stream, dev, w)), w)


def adam_grad_norm(plan: int, max_norm: float, norm, grad_scale, workspace, stream=None):
    """norm of all the plan's gradients and grad_scale = min(1, max_norm / norm), float32 CUDA tensors of one element; workspace as for EDQ."""
    w, (L, dev) = "collage_adam_grad_norm", _operators()
    ws, ws_bytes = _scratch(workspace, dev, w)
    _check(L.collage_adam_grad_norm(plan, max_norm, _vector(norm, _F32, 1, dev, w), _vector(grad_scale, _F32, 1, dev, w), ws, ws_bytes,
                                    _stream(stream, dev, w)), w)

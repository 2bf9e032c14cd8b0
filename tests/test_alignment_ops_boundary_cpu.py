"""Refusals of the block norm, the token losses and the multi-tensor AdamW step, all detected on the host before any CUDA call."""
import ctypes

import pytest

from paper_2405_03637_b200 import binding as B

A, SLOT = 0x100000, 0x100000                    # never dereferenced; arrays placed SLOT apart do not overlap
NAN, INF = float("nan"), float("inf")


def at(i):
    return A + i * SLOT


def mat(i, rows, cols, ld=None, offset=0):
    return B.Matrix(at(i) + offset, rows, cols, cols if ld is None else ld)


@pytest.fixture(scope="module")
def L():
    return B.lib()


def test_packed_structures_have_the_headers_layout():
    B._operators()
    assert ctypes.sizeof(B.BlockNorm) == 2 * 32 + len(B._pack_block_norm(0, 0, 0, 0, 0, 0)) == 112
    assert ctypes.sizeof(B.Tokens) == 32 + len(B._pack_tokens(0, 0, 0, 0)) == 56
    assert ctypes.sizeof(B.Policy) == len(B._pack_policy(*[0] * 7)) == 56
    assert ctypes.sizeof(B.Preference) == len(B._pack_preference(*[0] * 15)) == 112
    assert ctypes.sizeof(B.AdamTensor) == 64


def norm_in(block=mat(0, 4, 64), gate=mat(1, 1, 64), post=at(2), pre=at(3), eps=1e-6, alpha=1.0, beta=1.0, act=0):
    return B.BlockNorm(block, gate if gate is not None else B.Matrix(None, 0, 0, 0), post, pre, eps, alpha, beta, act)


def test_block_norm_refusals(L):
    def call(s=norm_in(), x=mat(4, 4, 64), r=mat(5, 4, 64), y=mat(6, 4, 64), y8=None, s8=None, rpost=at(8), rpre=at(9)):
        return L.collage_block_norm(s, x, r, y, y8, s8, rpost, rpre, None)
    assert call(s=None) == B.ERR_NULL and call(x=None) == B.ERR_NULL and call(r=None) == B.ERR_NULL
    assert call(y8=mat(7, 4, 64)) == B.ERR_NULL                           # 8 bits without a scale
    assert call(s8=at(7)) == B.ERR_ARG                                    # a scale without 8 bits
    assert call(s=norm_in(pre=None)) == B.ERR_NULL                        # y without the norm that makes it
    assert call(s=norm_in(pre=None), y=None) == B.ERR_ARG                 # rstd_pre without it
    assert call(s=norm_in(post=None)) == B.ERR_ARG                        # rstd_post without its norm
    for v in (-1e-6, NAN, INF):
        assert call(s=norm_in(eps=v)) == B.ERR_ARG
    for v in (NAN, INF, 1e39):
        assert call(s=norm_in(alpha=v)) == B.ERR_ARG and call(s=norm_in(beta=v)) == B.ERR_ARG
    assert call(s=norm_in(act=3)) == B.ERR_ARG and call(s=norm_in(act=-1)) == B.ERR_ARG
    assert call(s=norm_in(gate=mat(1, 2, 64))) == B.ERR_ARG               # neither one row nor a row for each
    assert call(s=norm_in(gate=mat(1, 1, 63))) == B.ERR_ARG
    assert call(s=norm_in(gate=mat(1, 4, 64, ld=63))) == B.ERR_ARG
    assert call(x=mat(4, 3, 64)) == B.ERR_ARG and call(y=mat(6, 4, 63)) == B.ERR_ARG
    assert call(x=mat(4, 4, 64, offset=1)) == B.ERR_ARG and call(s=norm_in(post=at(2) + 1)) == B.ERR_ARG and call(rpost=at(8) + 2) == B.ERR_ARG
    assert call(s=norm_in(block=B.Matrix(None, 4, 64, 64))) == B.ERR_NULL
    assert call(y=mat(5, 4, 64)) == B.ERR_ALIAS                           # two outputs in one place
    assert call(r=mat(4, 4, 64, offset=2)) == B.ERR_ALIAS                 # r over part of x
    assert call(y=mat(4, 4, 64)) == B.ERR_ALIAS                           # y over x
    assert call(r=mat(1, 4, 64)) == B.ERR_ALIAS                           # r over the gate
    assert call(rpre=at(2)) == B.ERR_ALIAS


def test_block_norm_backward_refusals(L):
    need = B.block_norm_workspace_bytes(64)
    assert need > 0

    def call(s=norm_in(), dy=mat(4, 4, 64), dr=mat(5, 4, 64), r=mat(6, 4, 64), rpost=at(7), rpre=at(8), dx=mat(9, 4, 64), do=mat(10, 4, 64),
             dg=mat(11, 1, 64), dpost=at(12), dpre=at(13), ws=at(14), nb=need):
        return L.collage_block_norm_backward(s, dy, dr, r, rpost, rpre, dx, do, dg, dpost, dpre, ws, nb, None)
    assert call(s=None) == B.ERR_NULL and call(dy=None, dr=None, dpre=None) == B.ERR_NULL
    assert call(dx=None, do=None, dg=None, dpost=None, dpre=None) == B.ERR_NULL
    assert call(r=None) == B.ERR_NULL and call(rpre=None) == B.ERR_NULL and call(rpost=None) == B.ERR_NULL and call(s=norm_in(pre=None)) == B.ERR_NULL
    assert call(dy=None) == B.ERR_ARG                                     # dpre_weight without a gradient of y
    assert call(s=norm_in(post=None)) == B.ERR_ARG and call(s=norm_in(gate=None)) == B.ERR_ARG
    assert call(ws=None) == B.ERR_WORKSPACE and call(nb=need - 1) == B.ERR_WORKSPACE and call(ws=at(14) + 8) == B.ERR_WORKSPACE
    assert call(ws=None, dpost=None, dpre=None) == B.ERR_WORKSPACE        # a gate of channels wants a sum too
    assert call(dg=mat(11, 4, 64)) == B.ERR_ARG and call(do=mat(10, 4, 63)) == B.ERR_ARG
    assert call(dx=mat(6, 4, 64)) == B.ERR_ALIAS                          # over r
    assert call(dx=mat(0, 4, 64)) == B.ERR_ALIAS                          # over the block's output
    assert call(dx=mat(4, 4, 64, offset=16)) == B.ERR_ALIAS               # over part of dy
    assert call(do=mat(9, 4, 64)) == B.ERR_ALIAS and call(dpost=at(13)) == B.ERR_ALIAS and call(ws=at(9)) == B.ERR_ALIAS
    assert call(dx=mat(4, 4, 64), do=mat(4, 4, 64)) == B.ERR_ALIAS        # both in dy's place


def tokens(z=mat(0, 6, 100), y=at(1), dtype=B.DTYPE_BF16, size=4, temp=1.0):
    return B.Tokens(z, y, dtype, size, temp)


def test_token_refusals(L):
    dz = mat(2, 6, 100)
    logp = lambda t, p=at(3), s=at(4), rest=at(5): L.collage_token_logp(t, p, rest, s, None)  # noqa: E731
    back = lambda t, s=at(4), g=at(3), d=dz: L.collage_token_logp_backward(t, s, g, d, None)  # noqa: E731
    assert logp(None) == B.ERR_NULL and logp(tokens(), p=None) == B.ERR_NULL and logp(tokens(y=None)) == B.ERR_NULL
    assert back(None) == B.ERR_NULL and back(tokens(), d=None) == B.ERR_NULL and back(tokens(), s=None) == B.ERR_NULL and back(tokens(), g=None) == B.ERR_NULL
    for f in (logp, back):
        assert f(tokens(dtype=2)) == B.ERR_ARG and f(tokens(size=2)) == B.ERR_ARG and f(tokens(y=at(1) + 2)) == B.ERR_ARG
        for temp in (0.0, -1.0, NAN, INF, 1e-60, 1e60):
            assert f(tokens(temp=temp)) == B.ERR_ARG
        assert f(tokens(size=8, y=at(1) + 4)) == B.ERR_ARG
        assert f(tokens(), s=at(4) + 4) == B.ERR_ARG                      # pairs of floats
        assert f(tokens(z=mat(0, 6, 100, ld=99))) == B.ERR_ARG
    assert logp(tokens(), s=at(3)) == B.ERR_ALIAS and logp(tokens(), rest=at(3)) == B.ERR_ALIAS and logp(tokens(), rest=at(5) + 2) == B.ERR_ARG and logp(tokens(), p=at(0)) == B.ERR_ALIAS
    assert back(tokens(), d=mat(2, 6, 99)) == B.ERR_ARG
    assert back(tokens(), d=mat(0, 6, 100, offset=2)) == B.ERR_ALIAS and back(tokens(), d=mat(3, 6, 100)) == B.ERR_ALIAS


def test_policy_refusals(L):
    def call(t=tokens(), old=at(3), ref=at(4), adv=at(5), w=at(6), low=0.2, high=0.2, klw=0.1, loss=at(7), logp=at(8), kl=at(9), d=mat(2, 6, 100), p=True):
        return L.collage_policy_loss_and_grad(t, B.Policy(old, ref, adv, w, low, high, klw) if p else None, loss, logp, kl, d, None)
    assert call(t=None) == B.ERR_NULL and call(p=False) == B.ERR_NULL
    for k in ("adv", "w", "loss", "d"):
        assert call(**{k: None}) == B.ERR_NULL
    for k, v in (("low", -0.1), ("low", 1.5), ("low", NAN), ("high", -0.1), ("high", NAN), ("klw", -1.0), ("klw", NAN), ("klw", INF), ("klw", 1e39)):
        assert call(**{k: v}) == B.ERR_ARG, (k, v)
    assert call(ref=None) == B.ERR_ARG and call(ref=None, kl=None) == B.ERR_ARG and call(ref=None, klw=0.0) == B.ERR_ARG
    assert call(adv=at(5) + 2) == B.ERR_ARG and call(logp=at(8) + 1) == B.ERR_ARG
    assert call(loss=at(6)) == B.ERR_ALIAS and call(kl=at(8)) == B.ERR_ALIAS and call(logp=at(3)) == B.ERR_ALIAS
    assert call(d=mat(5, 6, 100)) == B.ERR_ALIAS


def test_preference_refusals(L):
    def call(logp=at(0), rest=at(8), ref=at(1), y=at(2), o=at(3), w=at(4), rows=8, vocab=100, pairs=2, ysize=8, osize=4, beta=0.1, margin=0.0, smooth=0.0, loss=at(5),
             ratio=at(6), grad=at(7), s=True):
        p = B.Preference(logp, rest, ref, y, o, w, rows, vocab, pairs, ysize, osize, beta, margin, smooth, 0)
        return L.collage_preference_loss(ctypes.byref(p) if s else None, loss, ratio, grad, None)
    assert call(s=False) == B.ERR_NULL
    for k in ("logp", "y", "o", "loss"):
        assert call(**{k: None}) == B.ERR_NULL
    for k, v in (("beta", NAN), ("beta", 1e39), ("margin", INF), ("smooth", -0.1), ("smooth", 1.1), ("smooth", NAN), ("ysize", 2), ("osize", 1), ("logp", at(0) + 2), ("rest", at(8) + 1),
                 ("y", at(2) + 4), ("o", at(3) + 2), ("grad", at(7) + 1)):
        assert call(**{k: v}) == B.ERR_ARG, (k, v)
    for k in ("rows", "vocab", "pairs"):
        assert call(**{k: 1 << 31}) == B.ERR_LIMIT
    assert call(grad=at(0)) == B.ERR_ALIAS and call(grad=at(8)) == B.ERR_ALIAS and call(loss=at(4)) == B.ERR_ALIAS and call(ratio=at(5)) == B.ERR_ALIAS and call(grad=at(3)) == B.ERR_ALIAS


def adam_tensor(i=0, n=1000, state=B.STATE_E4M3, form=B.REST_BF16, **kw):
    codes = state == B.STATE_E4M3
    f = dict(theta=at(8 * i), rest=at(8 * i + 1) if form else None, m=at(8 * i + 2), v=at(8 * i + 3), m_scale=at(8 * i + 4) if codes else None,
             v_scale=at(8 * i + 5) if codes else None, grad=at(8 * i + 6), n=n)
    f.update(kw)
    return B.AdamTensor(*[f[k] for k in ("theta", "rest", "m", "v", "m_scale", "v_scale", "grad", "n")])


def test_adam_plan_refusals(L):
    def call(*tensors, num=None, state=B.STATE_E4M3, rest=B.REST_BF16, out=True):
        arr, plan = (B.AdamTensor * max(1, len(tensors)))(*tensors), ctypes.c_void_p(1)
        st = L.collage_adam_plan_create(arr if tensors else None, len(tensors) if num is None else num, state, rest, ctypes.byref(plan) if out else None)
        assert not out or st == B.OK or not plan.value                    # no plan comes of an error
        return st
    assert call(adam_tensor(), out=False) == B.ERR_NULL
    assert call(num=-1) == B.ERR_ARG and call(num=1) == B.ERR_NULL
    assert call(adam_tensor(), state=2) == B.ERR_ARG and call(adam_tensor(), rest=3) == B.ERR_ARG and call(adam_tensor(), rest=-1) == B.ERR_ARG
    for k in ("theta", "rest", "m", "v", "m_scale", "v_scale", "grad"):
        assert call(adam_tensor(), adam_tensor(1, **{k: None})) == B.ERR_NULL, k
    for k, off in (("theta", 1), ("rest", 1), ("grad", 1), ("m_scale", 2), ("v_scale", 1)):
        assert call(adam_tensor(**{k: at(40) + off})) == B.ERR_ARG, k
    f32 = dict(state=B.STATE_F32, rest=B.REST_F32)
    for k in ("m", "v", "rest"):
        assert call(adam_tensor(state=B.STATE_F32, **{k: at(40) + 2}), **f32) == B.ERR_ARG, k
    assert call(adam_tensor(state=B.STATE_F32, m_scale=at(40)), **f32) == B.ERR_ARG         # a scale that floats do not have
    assert call(adam_tensor(), rest=B.REST_NONE) == B.ERR_ARG                               # a second part that the form does not have
    assert call(adam_tensor(n=1 << 59)) == B.ERR_ARG and call(adam_tensor(n=1 << 45)) == B.ERR_ARG
    assert call(adam_tensor(), adam_tensor(1, grad=at(6) + 100)) == B.ERR_ALIAS             # gradients that overlap
    assert call(adam_tensor(v_scale=at(4) + 12)) == B.ERR_ALIAS                             # 1000 elements have four scales
    assert call(adam_tensor(m=at(3) - 999)) == B.ERR_ALIAS


def test_adam_calls_refuse(L):
    h = lambda lr=1e-3, b1=0.9, b2=0.999, eps=1e-8, wd=0.0, flags=0, edq=None: ctypes.byref(B.Hyper(lr, b1, b2, eps, wd, flags, edq, None, 0))  # noqa: E731
    assert L.collage_adam_step(None, h(), 1, 0, None, None) == B.ERR_NULL
    assert L.collage_adam_grad_norm(None, 1.0, at(0), at(1), at(2), 1 << 20, None) == B.ERR_NULL
    assert L.collage_adam_plan_destroy(None) == B.OK

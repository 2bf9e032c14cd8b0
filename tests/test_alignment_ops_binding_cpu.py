"""What the binding of the block norm, the token losses and the multi-tensor AdamW step refuses, without a GPU."""
import pytest
import torch

from paper_2405_03637_b200 import binding as B
from test_training_ops_binding_cpu import Calls, Fake, FakeStream, elsewhere

F32, E4M3, BF16 = torch.float32, torch.float8_e4m3fn, torch.bfloat16
ROW, COL, MAT = Fake(4, dtype=F32), Fake(64), Fake(4, 64)
LOGITS, TARGET = Fake(4, 99), Fake(4, dtype=torch.int64)
OPERATORS = {
    "block_norm": (B.block_norm, [MAT, MAT, MAT], dict(gate=Fake(1, 64), post_weight=COL, pre_weight=COL, y=MAT, y8=Fake(4, 64, dtype=E4M3), y8_scale=ROW,
                   rstd_post=ROW, rstd_pre=ROW)),
    "block_norm_backward": (B.block_norm_backward, [MAT, MAT, MAT, ROW, ROW, MAT, MAT], dict(dr=MAT, gate=MAT, post_weight=COL, pre_weight=COL, dgate=MAT,
                            dpost_weight=COL, dpre_weight=COL, workspace=Fake(64, dtype=torch.uint8))),
    "token_logp": (B.token_logp, [LOGITS, TARGET, 1.0, ROW], dict(stats=Fake(4, 2, dtype=F32), logp_rest=ROW)),
    "token_logp_backward": (B.token_logp_backward, [LOGITS, TARGET, 1.0, Fake(4, 2, dtype=F32), ROW, LOGITS], {}),
    "policy_loss_and_grad": (B.policy_loss_and_grad, [LOGITS, TARGET, 1.0, ROW, ROW, ROW, LOGITS], dict(old_logp=ROW, ref_logp=ROW, logp=ROW, kl=ROW)),
    "preference_loss": (B.preference_loss, [ROW, TARGET, 99, Fake(5, dtype=torch.int32), 0.1, Fake(2, dtype=F32)], dict(grad_logp=ROW, ref_logp=ROW, logp_rest=ROW,
                        pair_weight=Fake(2, dtype=F32), log_ratio=Fake(2, dtype=F32))),
    "adam_step": (B.adam_step, [0x7000, B.make_hyper(1e-3, 0.9, 0.999, 1e-8, 0.0), 1], dict(grad_scale=Fake(1, dtype=F32))),
    "adam_grad_norm": (B.adam_grad_norm, [0x7000, 1.0, Fake(1, dtype=F32), Fake(1, dtype=F32), Fake(64, dtype=torch.uint8)], {}),
}


@pytest.fixture
def calls(monkeypatch):
    B._operators()
    c = Calls()
    monkeypatch.setattr(B, "_packed", c)
    monkeypatch.setattr(B, "_current_device", lambda: 0, raising=False)
    monkeypatch.setattr(B, "_current_stream", lambda dev: 0, raising=False)
    return c


def refused(f, *args, status=B.ERR_ARG, **kwargs):
    with pytest.raises(B.CollageError) as e:
        f(*args, **kwargs)
    assert e.value.status == status


@pytest.mark.parametrize("name", OPERATORS)
def test_tensors_of_another_device_type_or_length_are_refused(calls, name):
    f, args, kwargs = OPERATORS[name]
    f(*args, **kwargs)
    assert calls.count == 1
    every = list(enumerate(args)) + list(kwargs.items())
    for key, t in every:
        if not isinstance(t, Fake):
            continue
        wrong = [elsewhere(t, 1), elsewhere(t, -1)]                       # another GPU; the host
        if t.dtype is not torch.uint8:
            wrong.append(Fake(*t.shape, dtype=torch.float16))
            if len(t.shape) == 1:
                wrong += [Fake(t.shape[0] + 1, dtype=t.dtype)] * (name != "preference_loss" or key not in (0, 3))
        for bad in wrong:
            refused(f, *[bad if i == key else a for i, a in enumerate(args)], **{k: bad if k == key else a for k, a in kwargs.items()})
    assert calls.count == 1


def test_tensors_of_one_device_that_is_not_the_current_one_are_refused(calls, monkeypatch):
    monkeypatch.setattr(B, "_current_device", lambda: 3, raising=False)
    for f, args, kwargs in OPERATORS.values():
        refused(f, *args, **kwargs)
    assert calls.count == 0


@pytest.mark.parametrize("name", OPERATORS)
def test_the_stream_has_to_be_named_where_another_than_the_default_is_current(calls, monkeypatch, name):
    f, args, kwargs = OPERATORS[name]
    monkeypatch.setattr(B, "_current_stream", lambda dev: 0x5000, raising=False)
    refused(f, *args, **kwargs)
    refused(f, *args, **kwargs, stream=FakeStream(0x5000, device=1))
    assert calls.count == 0
    f(*args, **kwargs, stream=FakeStream(0x5000))
    assert calls.count == 1


def test_missing_tensors_and_odd_numbers_of_offsets(calls):
    for name, at in (("block_norm", 0), ("block_norm", 1), ("block_norm", 2), ("token_logp", 0), ("token_logp", 1), ("preference_loss", 0), ("preference_loss", 3)):
        f, args, kwargs = OPERATORS[name]
        refused(f, *args[:at], None, *args[at + 1:], **kwargs, status=B.ERR_NULL)
    f, args, kwargs = OPERATORS["preference_loss"]
    refused(f, *args[:3], Fake(4, dtype=torch.int32), *args[4:], **kwargs)
    refused(f, *args[:3], Fake(0, dtype=torch.int32), *args[4:], **kwargs)
    assert calls.count == 0


class FakePlans:
    """Stands for the library where plans are made."""

    def __init__(self):
        self.made = []

    def collage_adam_plan_create(self, arr, num, state, rest, out):
        self.made.append((num, state, rest, [(t.n, t.rest, t.m_scale) for t in arr[:num]]))
        return B.OK

    def collage_status_string(self, status):
        return b"refused"


def test_adam_plan_takes_tensors_of_one_form(calls, monkeypatch):
    plans = FakePlans()
    monkeypatch.setattr(B, "lib", lambda: plans)

    def tensor(n=300, codes=True, rest=BF16, **kw):
        t = dict(theta=Fake(n), rest=rest and Fake(n, dtype=rest), m=Fake(n, dtype=E4M3 if codes else F32), v=Fake(n, dtype=E4M3 if codes else F32),
                 m_scale=Fake(-(-n // 256), dtype=F32) if codes else None, v_scale=Fake(-(-n // 256), dtype=F32) if codes else None, grad=Fake(n))
        t.update(kw)
        return tuple(t.values())
    B.adam_plan_create([tensor(), tensor(256)])
    B.adam_plan_create([tensor(codes=False, rest=None)])
    B.adam_plan_create([tensor(rest=F32)])
    B.adam_plan_create([])
    assert [p[:3] for p in plans.made] == [(2, B.STATE_E4M3, B.REST_BF16), (1, B.STATE_F32, B.REST_NONE), (1, B.STATE_E4M3, B.REST_F32), (0, 0, 0)]
    made = len(plans.made)
    for bad in ([tensor(), tensor(codes=False)], [tensor(), tensor(rest=None)], [tensor(), tensor(rest=F32)], [tensor(m=Fake(300, dtype=F32))],
                [tensor(m_scale=Fake(1, dtype=F32))], [tensor(grad=Fake(299))], [tensor(theta=Fake(300, dtype=F32))], [tensor(v=Fake(300, dtype=torch.uint8))],
                [tensor(theta=Fake(300, contiguous=False))], [tensor(theta=elsewhere(Fake(300), 1))], [tensor(rest=torch.float16)]):
        refused(B.adam_plan_create, bad)
    for k in ("theta", "m", "v", "grad"):
        refused(B.adam_plan_create, [tensor(**{k: None})], status=B.ERR_NULL)
    assert len(plans.made) == made

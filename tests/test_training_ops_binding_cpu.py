"""The binding of the training-step operators without a GPU: what it needs to be imported, and what it refuses."""
import subprocess
import sys
from pathlib import Path

import pytest
import torch

from paper_2405_03637_b200 import binding as B

ROOT = Path(__file__).resolve().parent.parent

WITHOUT_TORCH = """
import sys
sys.modules["torch"] = None                                  # any import of it raises
from paper_2405_03637_b200 import binding as B
assert B.derive_scalars(B.make_hyper(1e-3, 0.9, 0.999, 1e-8, 0.0), 1)["b1"] == 0x3F66
assert B.workspace_bytes() > 0 and B.rms_norm_workspace_bytes(64) > 0
"""


def test_the_binding_does_without_torch_but_for_the_operators():
    p = subprocess.run([sys.executable, "-c", WITHOUT_TORCH], cwd=ROOT, capture_output=True, text=True, timeout=120)
    assert p.returncode == 0, p.stderr[-2000:]


class Fake:
    """What the binding asks of a tensor, on a device of the test's choosing."""

    def __init__(self, *shape, dtype=torch.bfloat16, device=0, contiguous=True):
        self.shape, self.dtype, self.device, self.is_cuda, self.contiguous = torch.Size(shape), dtype, device, device >= 0, contiguous

    def get_device(self):
        return self.device

    def stride(self):
        return torch.empty(self.shape, device="meta").stride()

    def numel(self):
        return self.shape.numel()

    def element_size(self):
        return torch.empty(0, dtype=self.dtype).element_size()

    def is_contiguous(self):
        return self.contiguous

    def data_ptr(self):
        return 0x100000


class Calls:
    """Stands for the library: every call succeeds and is counted."""

    def __init__(self):
        self.count = 0

    def __getattr__(self, name):
        def call(*args):
            self.count += 1
            return B.OK
        return call


@pytest.fixture
def calls(monkeypatch):
    B._operators()
    c = Calls()
    monkeypatch.setattr(B, "_packed", c)
    monkeypatch.setattr(B, "_current_device", lambda: 0, raising=False)
    monkeypatch.setattr(B, "_current_stream", lambda dev: 0, raising=False)
    return c


F32, E4M3 = torch.float32, torch.float8_e4m3fn
OPERATORS = {
    "add_rms_norm": (B.add_rms_norm, [Fake(4, 64), Fake(4, 64), Fake(64)], dict(eps=1e-5, residual_out=Fake(4, 64), y=Fake(4, 64), y8=Fake(4, 64, dtype=E4M3),
                     y8_scale=Fake(4, dtype=F32), rstd=Fake(4, dtype=F32))),
    "add_rms_norm_backward": (B.add_rms_norm_backward, [Fake(4, 64), Fake(4, 64), Fake(4, dtype=F32), Fake(64), Fake(4, 64), Fake(64),
                              Fake(320 * 4 * 64, dtype=torch.uint8)], dict(dresidual=Fake(4, 64))),
    "quantize_rows": (B.quantize_rows, [Fake(4, 64), Fake(4, 64, dtype=E4M3), Fake(4, dtype=F32)], {}),
    "gated_ffn": (B.gated_ffn, [Fake(4, 64), Fake(8, 64), Fake(8, 64), Fake(4, 8)], dict(gate=Fake(4, 8), up=Fake(4, 8))),
    "gated_ffn_backward": (B.gated_ffn_backward, [Fake(4, 8), Fake(4, 64), Fake(8, 64), Fake(8, 64)] + [Fake(4, 8)] * 4,
                           dict(dx=Fake(4, 64), dw_gate=Fake(8, 64), dw_up=Fake(8, 64))),
    "gated_ffn_e4m3": (B.gated_ffn_e4m3, [Fake(4, 64, dtype=E4M3), Fake(4, dtype=F32), Fake(8, 64, dtype=E4M3), Fake(8, dtype=F32),
                       Fake(8, 64, dtype=E4M3), Fake(8, dtype=F32), Fake(4, 8)], {}),
    "distill_loss": (B.distill_loss, [Fake(4, 99), Fake(4, 3, dtype=torch.int32), Fake(4, 3, dtype=F32), 1.0, Fake(4, dtype=F32)], dict(lse=Fake(4, dtype=F32))),
    "distill_loss_backward": (B.distill_loss_backward, [Fake(4, 99), Fake(4, 3, dtype=torch.int64), Fake(4, 3, dtype=F32), 1.0, Fake(4, dtype=F32),
                              Fake(4, dtype=F32), Fake(4, 99)], {}),
    "distill_loss_and_grad": (B.distill_loss_and_grad, [Fake(4, 99), Fake(4, 3, dtype=torch.int32), Fake(4, 3, dtype=F32), 1.0, Fake(4, dtype=F32),
                              Fake(4, dtype=F32), Fake(4, 99)], {}),
}


def elsewhere(t, device):
    return Fake(*t.shape, dtype=t.dtype, device=device)


@pytest.mark.parametrize("name", OPERATORS)
def test_tensors_of_another_device_are_refused(calls, name):
    f, args, kwargs = OPERATORS[name]
    f(*args, **kwargs)
    assert calls.count == 1
    for device in (1, -1):                                   # another GPU; the host
        for i, t in enumerate(args):
            if isinstance(t, Fake):
                with pytest.raises(B.CollageError) as e:
                    f(*args[:i], elsewhere(t, device), *args[i + 1:], **kwargs)
                assert e.value.status == B.ERR_ARG
        for k, t in kwargs.items():
            if isinstance(t, Fake):
                with pytest.raises(B.CollageError) as e:
                    f(*args, **{**kwargs, k: elsewhere(t, device)})
                assert e.value.status == B.ERR_ARG
    assert calls.count == 1


def test_tensors_of_one_device_that_is_not_the_current_one_are_refused(calls, monkeypatch):
    monkeypatch.setattr(B, "_current_device", lambda: 3, raising=False)
    for f, args, kwargs in OPERATORS.values():
        with pytest.raises(B.CollageError) as e:
            f(*args, **kwargs)
        assert e.value.status == B.ERR_ARG
    assert calls.count == 0


def test_a_workspace_with_gaps_is_refused(calls):
    f, args, kwargs = OPERATORS["add_rms_norm_backward"]
    with pytest.raises(B.CollageError) as e:
        f(*args[:6], Fake(*args[6].shape, dtype=torch.uint8, contiguous=False), **kwargs)
    assert e.value.status == B.ERR_ARG and calls.count == 0


class FakeStream:
    def __init__(self, address, device=0):
        self.cuda_stream, self.device_index = address, device


@pytest.mark.parametrize("name", OPERATORS)
def test_the_stream_has_to_be_named_where_another_than_the_default_is_current(calls, monkeypatch, name):
    f, args, kwargs = OPERATORS[name]
    monkeypatch.setattr(B, "_current_stream", lambda dev: 0x5000, raising=False)

    def refused(stream):
        with pytest.raises(B.CollageError) as e:
            f(*args, **kwargs, stream=stream)
        assert e.value.status == B.ERR_ARG
    refused(None)
    refused(FakeStream(0x5000, device=1))
    assert calls.count == 0
    for stream in (FakeStream(0x5000), FakeStream(0), 0x5000, 0):      # the current one, the default one by its name, addresses
        f(*args, **kwargs, stream=stream)
    assert calls.count == 4

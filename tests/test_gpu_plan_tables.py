"""Plans are complete when their creation returns: a step may follow on any stream at once."""
import pytest
import torch

from paper_2405_03637_b200 import binding as B
from test_gpu_adam_multi import Tensor, hyper, workspace

pytestmark = pytest.mark.gpu


def collage_rows(n, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = (torch.randn(n, generator=g, device="cuda") * 0.02).to(torch.bfloat16)
    zeros = lambda: torch.zeros_like(x)  # noqa: E731
    return x, zeros(), zeros(), zeros(), zeros(), (torch.randn(n, generator=g, device="cuda") * 1e-3).to(torch.bfloat16), n


@pytest.mark.parametrize("kind", ["adam", "collage"])
def test_creation_waits_for_its_copies(kind):
    """The tables are copied on the default stream, behind whatever is under way there (a tenth of a second's kernel): nothing of it may be
    left when the call returns, or a step on another stream could read a table before it has arrived."""
    if kind == "adam":
        t = Tensor(70_001, B.STATE_E4M3, B.REST_BF16)
        make, destroy, rows = B.adam_plan_create, B.adam_plan_destroy, [t.row()]
    else:
        make, destroy, rows = B.plan_create, B.plan_destroy, [collage_rows(70_001, 3)]
    destroy(make(rows))                                                  # (allocations and first calls are behind us)
    torch.cuda.synchronize()
    torch.cuda._sleep(200_000_000)
    plan = make(rows)
    assert torch.cuda.default_stream().query()
    destroy(plan)


def test_a_step_on_another_stream_at_once():
    """Many plans, each stepped straight away on a stream that does not wait for the default one: the bits of a step after a synchronisation."""
    sizes = [70_001, 4096, 300] + [1 + 37 * i % 600 for i in range(500)]
    s = torch.cuda.Stream()
    for turn in range(4):
        sets = [[Tensor(n, B.STATE_E4M3, B.REST_BF16, seed=i + turn) for i, n in enumerate(sizes)] for _ in range(2)]
        flat = [collage_rows(70_001, turn) for _ in range(2)]
        ws, norms = [workspace() for _ in range(2)], [torch.zeros(1, device="cuda") for _ in range(2)]
        torch.cuda.synchronize()
        plans = []
        for k in range(2):
            plans.append((B.adam_plan_create([t.row() for t in sets[k]]), B.plan_create([flat[k]])))
            if k == 0:
                torch.cuda.synchronize()
            B.adam_grad_norm(plans[k][0], 1.0, norms[k], None, ws[k], stream=s)
            B.adam_step(plans[k][0], hyper(), 1, seed=5, stream=s)
            B.adamw_step_multi(plans[k][1], hyper(), 1, B.PLUS, stream=s)
            if k == 0:
                torch.cuda.synchronize()
        torch.cuda.synchronize()
        assert torch.equal(norms[0], norms[1])
        for a, b in zip(*sets):
            for x, y in zip(a.row(), b.row()):
                assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
        for x, y in zip(flat[0][:6], flat[1][:6]):
            assert torch.equal(x, y)
        for adam, collage in plans:
            B.adam_plan_destroy(adam)
            B.plan_destroy(collage)

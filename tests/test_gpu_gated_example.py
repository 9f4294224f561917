"""The gated form of the feed-forward example: its gradients against autograd in 32 bits, and the plans for both forms of its iteration."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
spec = importlib.util.spec_from_file_location("feed_forward", os.path.join(ROOT, "examples", "feed_forward.py"))
ff = importlib.util.module_from_spec(spec)
spec.loader.exec_module(ff)


@pytest.fixture(scope="module")
def setting():
    model = ff.GatedFeedForward(3, 200, 520, seed=3)
    gen = torch.Generator(device="cuda").manual_seed(4)
    x, target = (torch.randn(500, 200, generator=gen, device="cuda").bfloat16() for _ in range(2))
    return model, x, target


def autograd(model, x, target):
    p = {n: t.detach().float().cpu().requires_grad_() for n, t in model.p.items()}
    norm = lambda l, s: s * torch.rsqrt(s.square().mean(1, keepdim=True) + ff.EPS) * p[f"g.{l}"]
    s = x.float().cpu()
    for l in range(model.layers):
        g, u = (norm(l, s) @ p[f"w1.{l}"].t()).split(model.ffn, dim=1)
        s = s + (torch.nn.functional.silu(g) * u) @ p[f"w2.{l}"].t()
    loss = 0.5 * (norm(model.layers, s) - target.float().cpu()).square().sum(1).mean()
    loss.backward()
    return float(loss.detach()), {n: t.grad for n, t in p.items()}


@pytest.mark.parametrize("bits", [8, 16])
def test_gradients(setting, bits):
    """Each of the some ten tensors between a gradient and the loss is rounded to bf16 (2^-9 rms or less relative), each checkpoint to half
    a scale (about 1 % rms of a group): a few per cent together, where a wrong formula is off by all of it."""
    model, x, target = setting
    loss0, want = autograd(model, x, target)
    loss, got = model.iteration(x, target, kept_bits=bits)
    assert abs(float(loss) / loss0 - 1) < 0.01
    assert set(got) == set(want)
    for n, g in got.items():
        g0 = want[n]
        assert float((g.float().cpu() - g0).norm() / g0.norm()) < 0.05, n


def test_plans_of_the_recorded_iteration(setting):
    model, x, target = setting
    tas = {}
    for bits in (16, 8):
        rec = ff.Recorder()
        model.iteration(x, target, rec, bits)
        tas[bits] = rec.sequence()
        tas[bits].check()
    plans = {b: ff.plan(tas[b], 0) for b in tas}
    assert plans[8]["peak"] < plans[16]["peak"]
    assert all(r["planned"] <= r["peak"] for r in plans.values())
